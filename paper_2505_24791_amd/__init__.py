"""Thin Python binding of the HIP library ``libsjd.so`` (see ``include/sjd.h``).

Argument marshalling only: every step of selective Jacobi decoding runs in the library's kernels.
PyTorch is used for device memory and streams.  There is no CPU path: importing works anywhere,
but creating a ``Flow`` without the built library or without an MI355X raises.
"""
from __future__ import annotations

import ctypes as C
import os
from dataclasses import dataclass
from typing import Optional, Tuple

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libsjd.so")

SJD_OK, SJD_EINVAL, SJD_ENOMEM, SJD_EHIP, SJD_ENONFINITE, SJD_ESTATE = 0, -1, -2, -3, -4, -5
SJD_MAX_BLOCKS = 32
DTYPE_F32, DTYPE_BF16, DTYPE_F16 = 0, 1, 2
(PROF_GEMM, PROF_ATTENTION, PROF_EPILOGUE, PROF_DECODE_GEMM, PROF_DECODE_ATTN, PROF_OTHER, PROF_DECODE_FUSED,
 PROF_GEMM_RESID, PROF_GEMM_FC1, PROF_DECODE_RESID, PROF_GEMM_HEAD, PROF_DECODE_FC1, PROF_DECODE_HEAD) = range(13)
PROF_FAMILIES = 13
PROF_NAMES = ("gemm_qkv", "attention", "epilogue", "decode_qkv", "decode_attn", "other", "decode_fused", "gemm_resid",
              "gemm_fc1", "decode_resid", "gemm_head", "decode_fc1", "decode_head")
PROF_GEMM_ALL = (PROF_GEMM, PROF_GEMM_RESID, PROF_GEMM_FC1, PROF_GEMM_HEAD)            # every whole-sequence projection
PROF_DECODE_GEMM_ALL = (PROF_DECODE_GEMM, PROF_DECODE_RESID, PROF_DECODE_FC1, PROF_DECODE_HEAD)   # every single-token projection

EXPORTS = ("sjd_flow_create", "sjd_flow_load_weights", "sjd_jacobi_inverse_block", "sjd_sequential_inverse_block",
           "sjd_sample", "sjd_conditioner", "sjd_op_linear_h16", "sjd_jacobi_trace_block", "sjd_forward_block",
           "sjd_forward", "sjd_flow_set_mask_nearest", "sjd_flow_set_sequential_path", "sjd_flow_set_sequential_cus", "sjd_flow_set_projection_path",
           "sjd_op_panel_linear_h16", "sjd_op_panel_linear_h16_noalloc", "sjd_op_attention_h16", "sjd_op_qk_norm_rope", "sjd_op_kv4_write",
           "sjd_op_kv4_read", "sjd_op_kv4_attention", "sjd_kv4_attention_workspace", "sjd_profile_enable", "sjd_profile_read", "sjd_flow_device_bytes",
           "sjd_last_error", "sjd_flow_destroy")


class SjdConfig(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("n_blocks", "n_layers", "width", "n_heads", "mlp_ratio", "seq_len",
                                         "token_dim", "max_batch", "dtype")] + [("reverse_mask", C.c_uint32)]


class SjdJacobiOpts(C.Structure):
    _fields_ = [("tau", C.c_float), ("criterion", C.c_int32), ("init", C.c_int32), ("max_iters", C.c_int32),
                ("drop_converged", C.c_int32), ("refine_below", C.c_float)]


class SjdStats(C.Structure):
    _fields_ = [("block_iters", C.c_int32 * SJD_MAX_BLOCKS), ("mean_sample_iters", C.c_float * SJD_MAX_BLOCKS),
                ("block_ms", C.c_float * SJD_MAX_BLOCKS)]


class SjdProfile(C.Structure):
    _fields_ = [("ms", C.c_double * PROF_FAMILIES), ("launches", C.c_int64 * PROF_FAMILIES),
                ("flops", C.c_double * PROF_FAMILIES), ("bytes", C.c_double * PROF_FAMILIES)]


class SjdQkOpts(C.Structure):
    _fields_ = [("norm", C.c_int32), ("eps", C.c_float), ("q_gain", C.c_void_p), ("q_shift", C.c_void_p), ("k_gain", C.c_void_p),
                ("k_shift", C.c_void_p), ("rot_dim", C.c_int32), ("pairing", C.c_int32), ("n_axes", C.c_int32),
                ("axis_pairs", C.c_int32 * 4), ("freq", C.c_void_p)]


class SjdKv4(C.Structure):
    _fields_ = [("pages", C.c_void_p), ("n_pages", C.c_int32), ("n_kv_heads", C.c_int32), ("head_dim", C.c_int32), ("dtype", C.c_int32)]


class SjdKv4Attention(C.Structure):
    _fields_ = [("q", C.c_void_p), ("o", C.c_void_p), ("q_stride", C.c_int64), ("o_stride", C.c_int64), ("table_stride", C.c_int64),
                ("q_start", C.c_void_p), ("kv_len", C.c_void_p), ("page_table", C.c_void_p),
                ("n_seqs", C.c_int32), ("n_heads", C.c_int32), ("n_rows", C.c_int32), ("max_pages", C.c_int32), ("max_q", C.c_int32),
                ("max_kv", C.c_int32), ("causal", C.c_int32), ("skip_nearest", C.c_int32), ("window", C.c_int32), ("scale", C.c_float),
                ("workspace", C.c_void_p), ("workspace_bytes", C.c_size_t)]


class SjdError(RuntimeError):
    def __init__(self, code: int, msg: str):
        super().__init__(f"sjd error {code}: {msg}")
        self.code = code


_lib = None


def load_library() -> C.CDLL:
    """Loads libsjd.so; raises if it has not been built (there is no fallback)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise RuntimeError(f"{LIB_PATH} is missing: run `python -m paper_2505_24791_amd.build` "
                           "(or __graft_entry__.build()) first; this package has no CPU fallback")
    lib = C.CDLL(LIB_PATH)
    vp, i32p, fp = C.c_void_p, C.POINTER(C.c_int32), C.c_void_p
    lib.sjd_flow_create.argtypes = [C.POINTER(SjdConfig), C.POINTER(vp)]
    lib.sjd_flow_load_weights.argtypes = [vp, vp, C.c_size_t]
    lib.sjd_jacobi_inverse_block.argtypes = [vp, C.c_int, fp, fp, C.c_int, C.POINTER(SjdJacobiOpts), i32p, i32p, vp]
    lib.sjd_sequential_inverse_block.argtypes = [vp, C.c_int, fp, fp, C.c_int, vp]
    lib.sjd_sample.argtypes = [vp, fp, fp, C.c_int, C.c_uint32, C.POINTER(SjdJacobiOpts), C.POINTER(SjdStats), i32p, vp]
    lib.sjd_conditioner.argtypes = [vp, C.c_int, fp, fp, fp, C.c_int, vp]
    lib.sjd_jacobi_trace_block.argtypes = [vp, C.c_int, vp, vp, vp, C.c_int, C.POINTER(SjdJacobiOpts),
                                           C.POINTER(C.c_float), C.POINTER(C.c_float), C.POINTER(C.c_int32),
                                           C.POINTER(C.c_int32), vp]
    lib.sjd_forward_block.argtypes = [vp, C.c_int, vp, vp, vp, C.c_int, C.c_int, vp]
    lib.sjd_forward.argtypes = [vp, vp, vp, vp, C.c_int, vp]
    lib.sjd_flow_set_sequential_path.argtypes = [vp, C.c_int]
    lib.sjd_flow_set_sequential_cus.argtypes = [vp, C.c_int]
    lib.sjd_flow_set_mask_nearest.argtypes = [vp, C.c_int]
    lib.sjd_op_linear_h16.argtypes = [C.c_int, C.c_int, vp, vp, vp, vp, vp, C.c_int, C.c_int, C.c_int, C.c_int, vp]
    lib.sjd_op_attention_h16.argtypes = [C.c_int, vp, vp, C.c_int, C.c_int, C.c_int, vp]
    lib.sjd_op_qk_norm_rope.argtypes = [C.c_int, vp, vp, vp, C.c_int64, C.c_int, vp, C.c_int64, C.c_int, C.c_int, vp, C.c_int64, vp,
                                        C.c_int64, C.c_int, vp]
    lib.sjd_op_kv4_write.argtypes = [vp, vp, vp, C.c_int64, vp, C.c_int64, C.c_int, vp, vp, vp, C.c_int64, C.c_int, vp, C.c_int64, vp]
    lib.sjd_op_kv4_read.argtypes = [vp, vp, vp, C.c_int64, vp, C.c_int64, C.c_int, vp]
    lib.sjd_op_kv4_attention.argtypes = [vp, vp, vp]
    lib.sjd_kv4_attention_workspace.argtypes = [vp, vp, vp]
    lib.sjd_profile_enable.argtypes = [vp, C.c_uint32]
    lib.sjd_profile_read.argtypes = [vp, C.POINTER(SjdProfile), C.c_int]
    lib.sjd_flow_device_bytes.argtypes = [vp]
    lib.sjd_flow_device_bytes.restype = C.c_size_t
    lib.sjd_last_error.restype = C.c_char_p
    lib.sjd_flow_destroy.argtypes = [vp]
    lib.sjd_flow_destroy.restype = None
    for name in EXPORTS:
        if name not in ("sjd_flow_device_bytes", "sjd_last_error", "sjd_flow_destroy"):
            getattr(lib, name).restype = C.c_int
    _lib = lib
    return lib


def _check(rc: int, allow_nonfinite: bool = False) -> int:
    if rc == SJD_OK or (allow_nonfinite and rc == SJD_ENONFINITE):
        return rc
    raise SjdError(rc, load_library().sjd_last_error().decode())


@dataclass
class JacobiOpts:
    tau: float = 1e-3
    criterion: int = 0
    init: int = 0
    max_iters: int = 0
    drop_converged: int = 1
    refine_below: float = 0.0

    def c(self) -> SjdJacobiOpts:
        return SjdJacobiOpts(self.tau, self.criterion, self.init, self.max_iters, self.drop_converged,
                             self.refine_below)


def _stream_ptr() -> Optional[int]:
    import torch
    return C.c_void_p(torch.cuda.current_stream().cuda_stream)


def _dev(t, shape=None) -> C.c_void_p:
    import torch
    assert t.is_cuda and t.dtype == torch.float32 and t.is_contiguous(), "need a contiguous float32 CUDA tensor"
    if shape is not None:
        assert tuple(t.shape) == tuple(shape), (tuple(t.shape), tuple(shape))
    return C.c_void_p(t.data_ptr())


def op_linear_h16(a, wt, bias, M, N, K, epilogue, *, resid=None, kernel=0):
    """``sjd_op_linear_h16`` on torch tensors: a [M,K] and wt [N_pad,K] in float16 or bfloat16 (same
    type), bias [N] float32; returns c [M,N] (16-bit) or, for epilogue 2, updates ``resid`` in place."""
    import torch
    lib = load_library()
    assert a.is_cuda and wt.is_cuda and a.dtype == wt.dtype and a.is_contiguous() and wt.is_contiguous()
    assert wt.shape[0] % 256 == 0 and wt.shape[0] >= N and wt.shape[1] == K and tuple(a.shape) == (M, K)
    dtype = DTYPE_F16 if a.dtype == torch.float16 else DTYPE_BF16
    c = None
    if epilogue == 2:
        assert resid is not None and resid.dtype == torch.float32 and tuple(resid.shape) == (M, N) and resid.is_contiguous()
    else:
        c = torch.empty((M, N), dtype=a.dtype, device=a.device)
    _check(lib.sjd_op_linear_h16(dtype, kernel, C.c_void_p(a.data_ptr()), C.c_void_p(wt.data_ptr()),
                                 C.c_void_p(bias.data_ptr()), C.c_void_p(resid.data_ptr()) if resid is not None else None,
                                 C.c_void_p(c.data_ptr()) if c is not None else None, M, N, K, epilogue, _stream_ptr()))
    return resid if epilogue == 2 else c


def op_panel_linear_h16(a, wt, bias, M, N, epilogue, *, K=512, ln_g=None, ln_b=None, resid=None, noalloc=False):
    """``sjd_op_panel_linear_h16`` on torch tensors.  epilogue 0 / 1 (K = 512): a [M,512] float32, ln_g / ln_b
    [512] float32, returns c [M,N] in wt's type; epilogue 2: a [M,K] 16-bit, updates ``resid`` in place."""
    import torch
    lib = load_library()
    assert a.is_cuda and wt.is_cuda and a.is_contiguous() and wt.is_contiguous() and tuple(a.shape) == (M, K)
    assert wt.shape[0] >= N and wt.shape[1] == K and wt.dtype in (torch.float16, torch.bfloat16)
    dtype = DTYPE_F16 if wt.dtype == torch.float16 else DTYPE_BF16
    c = None
    if epilogue == 2:
        assert a.dtype == wt.dtype
        assert resid is not None and resid.dtype == torch.float32 and tuple(resid.shape) == (M, N) and resid.is_contiguous()
    else:
        assert a.dtype == torch.float32 and ln_g is not None and ln_b is not None
        c = torch.empty((M, N), dtype=wt.dtype, device=a.device)
    ptr = lambda t: C.c_void_p(t.data_ptr()) if t is not None else None
    fn = lib.sjd_op_panel_linear_h16_noalloc if noalloc else lib.sjd_op_panel_linear_h16
    _check(fn(dtype, ptr(a), ptr(ln_g), ptr(ln_b), ptr(wt), ptr(bias), ptr(resid), ptr(c), M, N, K, epilogue, _stream_ptr()))
    return resid if epilogue == 2 else c


def op_attention_h16(qkv, n_samples, T, H):
    """``sjd_op_attention_h16`` on a torch tensor: qkv [n_samples*T, 3*H*64] float16, bfloat16 or float32;
    returns o [n_samples*T, H*64] of the same type."""
    import torch
    lib = load_library()
    assert qkv.is_cuda and qkv.is_contiguous() and tuple(qkv.shape) == (n_samples * T, 3 * H * 64)
    dtype = {torch.float16: DTYPE_F16, torch.bfloat16: DTYPE_BF16, torch.float32: DTYPE_F32}[qkv.dtype]
    o = torch.empty((n_samples * T, H * 64), dtype=qkv.dtype, device=qkv.device)
    _check(lib.sjd_op_attention_h16(dtype, C.c_void_p(qkv.data_ptr()), C.c_void_p(o.data_ptr()), n_samples, T, H,
                                    _stream_ptr()))
    return o


KV4_PAGE = 64          # tokens of a page of the 4-bit cache
_MOST = 2 ** 31 - 1    # the library counts in 32 bits, and ctypes drops the others without a word
_NORMS = {None: 0, "none": 0, "rms": 1, "layer": 2}
_rt = None             # what the calls below use of the library and of torch, once both are loaded


def _runtime():
    global _rt
    import torch
    dtypes = {torch.float16: DTYPE_F16, torch.bfloat16: DTYPE_BF16, torch.float32: DTYPE_F32}
    # torch.cuda.current_stream() makes two objects around this number: 2.6 us of a call that takes 8
    _rt = (load_library(), torch._C._cuda_getCurrentRawStream, torch._C._cuda_getDevice, torch.cuda.device, torch.int32, dtypes)
    return _rt


def _refuse(what: str):
    raise SjdError(SJD_EINVAL, what)


def _row_dtype(torch_dtype) -> int:
    code = (_rt or _runtime())[5].get(torch_dtype)
    if code is None:
        _refuse(f"rows must be float16, bfloat16 or float32, not {torch_dtype}")
    return code


# The checks of the calls below run for every token of a serving loop: messages are made only where one fails, and a tensor that a call
# made itself is not looked at again.
def _rows3(t, what: str, dtype, device: int):
    """Shape and row stride of t [rows, heads, head_dim], the heads of a row following one another."""
    shape, stride = t.shape, t.stride()
    if t.dtype is not dtype or t.get_device() != device or len(shape) != 3:
        _refuse(f"{what}: need a {dtype} tensor [rows, heads, head_dim] on cuda:{device}")
    if ((stride[1] != shape[2] and shape[1] != 1) or (stride[2] != 1 and shape[2] != 1)) and shape[0]:
        _refuse(f"{what}: the heads of a row must follow one another")
    return shape, stride[0]


def _into(out, like, shape, dtype, what: str, device: int):
    """(out, its row stride): a new tensor, or the one that the caller gave, checked."""
    if out is None:
        return like.new_empty(shape, dtype=dtype), shape[1] * shape[2]
    got, stride = _rows3(out, what, dtype, device)
    if got != shape:
        _refuse(f"{what}: need the shape {tuple(shape)}")
    return out, stride


def _ints(t, what: str, shape, device: int) -> int:
    if t is None or t.dtype is not _rt[4] or t.get_device() != device or t.shape != shape or not t.is_contiguous():
        _refuse(f"{what}: need a contiguous int32 tensor {tuple(shape)} on cuda:{device}")
    return t.data_ptr()


def _launch(device: int, fn, *args) -> None:
    """Calls fn(*args, stream) with the tensors' device current, on that device's current stream."""
    stream = _rt[1](device)
    if device == _rt[2]():
        rc = fn(*args, stream)
    else:
        with _rt[3](device):
            rc = fn(*args, stream)
    if rc:
        _check(rc)


class QkOpts:
    """Norms and rotation of queries and keys (``sjd_qk_opts``), made once and used by many calls; it holds on to its tensors, and a call reads
    them where they are then (a captured graph where they were when it was captured).

    ``norm``: "none", "rms" or "layer" over the channels of a head, with gains and shifts [head_dim] float32 or None.  ``axis_pairs``: how
    many channel pairs each axis of the positions turns, together ``rot_dim / 2``; ``freq`` [rot_dim / 2] float32: radians per step of
    position.  ``adjacent``: pairs are (2i, 2i+1) instead of (i, i + rot_dim / 2)."""

    def __init__(self, *, norm: Optional[str] = "rms", eps: float = 1e-6, q_gain=None, q_shift=None, k_gain=None, k_shift=None,
                 rot_dim: int = 0, adjacent: bool = False, axis_pairs: Tuple[int, ...] = (), freq=None):
        if norm not in _NORMS:
            _refuse(f"norm must be one of {[n for n in _NORMS if n]}")
        if rot_dim and (not 1 <= len(axis_pairs) <= 4 or freq is None):
            _refuse("a rotation needs axis_pairs of 1 to 4 axes and freq")
        if rot_dim and (min(axis_pairs) < 0 or sum(axis_pairs) != rot_dim // 2):
            _refuse("axis_pairs must not be negative and add up to rot_dim / 2")
        vectors = {"q_gain": q_gain, "q_shift": q_shift, "k_gain": k_gain, "k_shift": k_shift, "freq": freq}
        self.vectors = {name: t for name, t in vectors.items() if t is not None}
        self.n_axes = len(axis_pairs) if rot_dim else 0
        self.c = SjdQkOpts(_NORMS[norm], eps, None, None, None, None, rot_dim, 1 if adjacent else 0, self.n_axes,
                           (C.c_int32 * 4)(*axis_pairs[:4]), None)
        self.address = C.addressof(self.c)
        self._take()

    def _take(self) -> None:
        """Checks the vectors and puts their addresses into the struct."""
        import torch
        held, at = list(self.vectors.values()), []
        for name, t in self.vectors.items():
            if not (t.is_cuda and t.dtype == torch.float32 and t.is_contiguous() and t.dim() == 1):
                _refuse(f"{name}: need a contiguous float32 vector on the GPU")
            at.append(t.data_ptr())
            if t.numel() and not at[-1]:
                _refuse(f"{name}: its memory has been freed")
        freq = self.vectors.get("freq")
        if freq is not None and freq.numel() != self.c.rot_dim // 2:
            _refuse("freq: need rot_dim / 2 values")
        sizes = {t.numel() for name, t in self.vectors.items() if name != "freq"}
        devices = {t.get_device() for t in self.vectors.values()}
        if len(sizes) > 1 or len(devices) > 1:
            _refuse("gains and shifts need one size, and all vectors one device")
        self.head_dim = sizes.pop() if sizes else None      # None: any
        self.device = devices.pop() if devices else None
        for name, address in zip(self.vectors, at):
            setattr(self.c, name, address)
        self._held, self._at = held, at

    def _for(self, head_dim: int, device: int) -> int:
        """The struct's address, for rows of this head size on this device."""
        if [t.data_ptr() for t in self._held] != self._at:  # a storage was replaced: the old one may be anyone's by now
            self._take()
        if (self.head_dim is not None and self.head_dim != head_dim) or (self.device is not None and self.device != device):
            _refuse(f"the options hold vectors of {self.head_dim} values on cuda:{self.device}, the rows are of {head_dim} on cuda:{device}")
        return self.address


def op_qk_norm_rope(q, k, pos, opts: QkOpts, *, q_out=None, k_out=None):
    """``sjd_op_qk_norm_rope``: q [rows, heads, head_dim] and k [rows, kv_heads, head_dim] (either may be None; views of a fused projection's
    rows as they are), pos [rows, axes] int32 (None without a rotation).  Returns (q_out, k_out), new tensors unless given; an output
    may be its input."""
    some = q if q is not None else k
    if some is None:
        _refuse("need q or k")
    dtype, device = some.dtype, some.get_device()
    if device < 0:         # host memory: options without vectors, and the other tensors of the call, would agree with it
        _refuse("need rows on the GPU")
    code = _row_dtype(dtype)
    qp = qs = qh = qo = qos = kp = ks = kh = ko = kos = 0
    if q is not None:
        shape, qs = _rows3(q, "q", dtype, device)
        n, qh, dim = shape
        q_out, qos = _into(q_out, q, shape, dtype, "q_out", device)
        qp, qo = q.data_ptr(), q_out.data_ptr()
    if k is not None:
        shape, ks = _rows3(k, "k", dtype, device)
        if q is not None and (shape[0] != n or shape[2] != dim):
            _refuse("k: other rows or another head size than q")
        n, kh, dim = shape
        k_out, kos = _into(k_out, k, shape, dtype, "k_out", device)
        kp, ko = k.data_ptr(), k_out.data_ptr()
    if n | qh | kh | dim > _MOST:
        _refuse("too many rows for one call")
    p = _ints(pos, "pos", (n, opts.n_axes), device) if opts.n_axes else None
    _launch(device, _rt[0].sjd_op_qk_norm_rope, code, opts._for(dim, device), p, qp, qs, qh, kp, ks, kh, dim, qo, qos, ko, kos, n)
    return q_out, k_out


class Kv4Cache:
    """A key/value cache of one layer in 4 bits (``sjd_kv4``): ``pages`` uint8 [pages, kv_heads, 68 * head_dim], 64 tokens to a page, of rows
    of ``dtype``.  The pages are the caller's: any tensor of that shape, e.g. ``Kv4Cache.zeros(...)``.  A call takes ``pages`` as it is then."""

    def __init__(self, pages, dtype):
        self.pages, self.dtype = pages, dtype
        self.c = SjdKv4(None, 0, 0, 0, _row_dtype(dtype))
        self.address = C.addressof(self.c)
        self._take()

    def _take(self) -> None:
        import torch
        pages = self.pages
        if not (pages.is_cuda and pages.dtype == torch.uint8 and pages.is_contiguous() and pages.dim() == 3 and pages.shape[2] % 68 == 0):
            _refuse("pages: need a contiguous uint8 tensor [pages, kv_heads, 68 * head_dim] on the GPU")
        self.device = pages.get_device()
        self.n_pages, self.kv_heads, self.head_dim = pages.shape[0], pages.shape[1], pages.shape[2] // 68
        c = self.c
        self._from, self._at = pages, pages.data_ptr()
        c.pages, c.n_pages, c.n_kv_heads, c.head_dim = self._at, self.n_pages, self.kv_heads, self.head_dim

    def _now(self) -> int:
        """The struct's address, for the pages as they are."""
        if self.pages is not self._from or self._from.data_ptr() != self._at:      # replaced: the old memory may be anyone's by now
            self._take()
        return self.address

    @classmethod
    def zeros(cls, n_pages: int, kv_heads: int, head_dim: int, dtype, device="cuda"):
        import torch
        return cls(torch.zeros((n_pages, kv_heads, 68 * head_dim), dtype=torch.uint8, device=device), dtype)

    def _kv(self, t, what: str, n: int):
        shape, stride = _rows3(t, what, self.dtype, self.device)
        if shape != (n, self.kv_heads, self.head_dim):
            _refuse(f"{what}: need [{n}, {self.kv_heads}, {self.head_dim}]")
        return t.data_ptr(), stride


def op_kv4_write(cache: Kv4Cache, k, v, slot, *, opts: Optional[QkOpts] = None, pos=None, q=None, q_out=None):
    """``sjd_op_kv4_write``: rows k, v [rows, kv_heads, head_dim] become the tokens ``slot`` [rows] int32 (page * 64 + offset; -1: left out).
    With ``opts`` the keys are normed and rotated first, and with ``q`` [rows, heads, head_dim] the queries of those rows too: returns them
    (``q_out`` or a new tensor), else None."""
    to = cache._now()
    n, device, dim = k.shape[0], cache.device, cache.head_dim
    (kp, ks), (vp_, vs) = cache._kv(k, "k", n), cache._kv(v, "v", n)
    sp = _ints(slot, "slot", (n,), device)
    op = pp = qp = qo = None
    qs = qos = heads = 0
    if opts is not None:
        op = opts._for(dim, device)
        if opts.n_axes:
            pp = _ints(pos, "pos", (n, opts.n_axes), device)
    if q is not None:
        if opts is None:
            _refuse("queries need opts")
        shape, qs = _rows3(q, "q", cache.dtype, device)
        if shape[0] != n or shape[2] != dim:
            _refuse("q: other rows or another head size")
        q_out, qos = _into(q_out, q, shape, cache.dtype, "q_out", device)
        qp, heads, qo = q.data_ptr(), shape[1], q_out.data_ptr()
    if n | heads > _MOST:
        _refuse("too many rows for one call")
    _launch(device, _rt[0].sjd_op_kv4_write, to, sp, kp, ks, vp_, vs, n, op, pp, qp, qs, heads, qo, qos)
    return q_out if q is not None else None


def op_kv4_read(cache: Kv4Cache, slot, *, k_out=None, v_out=None):
    """``sjd_op_kv4_read``: the tokens ``slot`` [rows] int32 of the cache, (k, v) [rows, kv_heads, head_dim]; zeros for a slot outside it."""
    held, n, device = cache._now(), slot.shape[0], cache.device
    sp = _ints(slot, "slot", (n,), device)
    if n > _MOST:
        _refuse("slot: too many rows for one call")
    shape = (n, cache.kv_heads, cache.head_dim)
    k_out, ks = _into(k_out, cache.pages, shape, cache.dtype, "k_out", device)
    v_out, vs = _into(v_out, cache.pages, shape, cache.dtype, "v_out", device)
    _launch(device, _rt[0].sjd_op_kv4_read, held, sp, k_out.data_ptr(), ks, v_out.data_ptr(), vs, n)
    return k_out, v_out


def op_kv4_attention(cache: Kv4Cache, q, page_table, kv_len, *, q_start=None, max_q: int = 1, max_kv: Optional[int] = None,
                     causal: bool = True, skip_nearest: int = 0, window: int = 0, scale: Optional[float] = None, out=None):
    """``sjd_op_kv4_attention``: q [rows, heads, head_dim], the last tokens of sequences with ``kv_len`` [seqs] int32 cached keys on the pages
    page_table [seqs, max_pages] int32; sequence b has the rows q_start[b] .. q_start[b+1] - 1 (q_start [seqs + 1] int32; None: max_q
    each).  max_q and max_kv bound the rows and keys of a sequence (max_kv None: all that the table has room for).  Rows of no
    sequence are left as they are in ``out`` (None: a new tensor, which holds anything there; ``q`` itself: in place)."""
    held, device = cache._now(), cache.device
    shape, q_stride = _rows3(q, "q", cache.dtype, device)
    n, heads, dim = shape
    if dim != cache.head_dim:
        _refuse("q: another head size than the cache's")
    table_shape, table_stride = page_table.shape, page_table.stride()
    if page_table.dtype is not _rt[4] or page_table.get_device() != device or len(table_shape) != 2 or (table_shape[1] > 1 and table_stride[1] != 1):
        _refuse(f"page_table: need int32 rows [seqs, max_pages] on cuda:{device}")
    seqs, pages = table_shape
    lens = _ints(kv_len, "kv_len", (seqs,), device)
    start = _ints(q_start, "q_start", (seqs + 1,), device) if q_start is not None else None
    out, out_stride = _into(out, q, shape, cache.dtype, "out", device)
    if max_kv is None:
        max_kv = pages * KV4_PAGE
    if n | heads | seqs | pages > _MOST:
        _refuse("too many rows, sequences or pages for one call")
    if not 0 <= max_q | max_kv | skip_nearest | window <= _MOST:
        _refuse("max_q, max_kv, skip_nearest and window are non-negative 32-bit integers")
    a = SjdKv4Attention(q.data_ptr(), out.data_ptr(), q_stride, out_stride, table_stride[0], start, lens, page_table.data_ptr(),
                        seqs, heads, n, pages, max_q, max_kv, 1 if causal else 0, skip_nearest,
                        window, dim ** -0.5 if scale is None else scale, None, 0)
    lib = _rt[0]
    address, need = C.addressof(a), C.c_size_t()
    rc = lib.sjd_kv4_attention_workspace(held, address, C.addressof(need))
    if rc:
        _check(rc)
    if need.value:
        workspace = cache.pages.new_empty(need.value)
        a.workspace, a.workspace_bytes = workspace.data_ptr(), need.value
    _launch(device, lib.sjd_op_kv4_attention, held, address)
    return out


class Flow:
    """A flow on the current device.  ``cfg`` needs the attributes of ``workloads.FlowConfig``."""

    def __init__(self, cfg, max_batch: Optional[int] = None, dtype: Optional[int] = None):
        self.lib = load_library()
        self.cfg = cfg
        self.max_batch = int(max_batch if max_batch is not None else cfg.batch)
        # 16-bit workloads default to IEEE-half operands: their bf16-valued weights convert exactly and
        # the activations keep three more mantissa bits, which the stopping rule needs (tau ~ 1e-3)
        self.dtype = (DTYPE_F16 if cfg.bf16 else DTYPE_F32) if dtype is None else dtype
        c = SjdConfig(cfg.n_blocks, cfg.n_layers, cfg.width, cfg.n_heads, cfg.mlp_ratio, cfg.seq_len, cfg.token_dim,
                      self.max_batch, self.dtype, cfg.reverse_mask)
        h = C.c_void_p()
        _check(self.lib.sjd_flow_create(C.byref(c), C.byref(h)))
        self._h = h

    def close(self) -> None:
        if getattr(self, "_h", None):
            self.lib.sjd_flow_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    @property
    def device_bytes(self) -> int:
        return int(self.lib.sjd_flow_device_bytes(self._h))

    def load_weights(self, blob: np.ndarray) -> None:
        blob = np.ascontiguousarray(blob, dtype=np.float32)
        _check(self.lib.sjd_flow_load_weights(self._h, C.c_void_p(blob.ctypes.data), blob.nbytes))

    def _shape(self, batch):
        return (batch, self.cfg.seq_len, self.cfg.token_dim)

    def conditioner(self, block: int, x):
        import torch
        B = x.shape[0]
        mu = torch.empty_like(x); al = torch.empty_like(x)
        _check(self.lib.sjd_conditioner(self._h, block, _dev(x, self._shape(B)), _dev(mu), _dev(al), B, _stream_ptr()))
        return mu, al

    def jacobi_inverse_block(self, block: int, z, opts: JacobiOpts, allow_nonfinite: bool = False, x0=None):
        """Returns (x, iters_per_sample int32 [B], passes_launched, rc).  With opts.init == 2 the first
        iterate is ``x0`` (copied, not modified)."""
        import torch
        B = z.shape[0]
        x = torch.empty_like(z) if x0 is None else x0.detach().clone().contiguous()
        iters = np.zeros(B, np.int32)
        passes = C.c_int32(0)
        o = opts.c()
        rc = _check(self.lib.sjd_jacobi_inverse_block(self._h, block, _dev(z, self._shape(B)), _dev(x), B, C.byref(o),
                                                      iters.ctypes.data_as(C.POINTER(C.c_int32)), C.byref(passes),
                                                      _stream_ptr()), allow_nonfinite)
        return x, iters, int(passes.value), rc

    def jacobi_trace_block(self, block: int, z, opts: JacobiOpts, x_ref=None, x0=None):
        """Jacobi decoding with the per-pass record.  Returns (x, iters [B], passes, delta [passes, B],
        err [passes, B] or None)."""
        import torch
        B = z.shape[0]
        T = self.cfg.seq_len
        cap = opts.max_iters if 0 < opts.max_iters < T else T
        x = torch.empty_like(z) if x0 is None else x0.detach().clone().contiguous()
        iters = np.zeros(B, np.int32)
        passes = C.c_int32(0)
        delta = np.zeros((cap, B), np.float32)
        err = np.zeros((cap, B), np.float32) if x_ref is not None else None
        o = opts.c()
        fp = C.POINTER(C.c_float)
        _check(self.lib.sjd_jacobi_trace_block(
            self._h, block, _dev(z, self._shape(B)), _dev(x), _dev(x_ref, self._shape(B)) if x_ref is not None else None,
            B, C.byref(o), delta.ctypes.data_as(fp), err.ctypes.data_as(fp) if err is not None else None,
            iters.ctypes.data_as(C.POINTER(C.c_int32)), C.byref(passes), _stream_ptr()))
        n = int(passes.value)
        return x, iters, n, delta[:n], (err[:n] if err is not None else None)

    def forward_block(self, block: int, x, logdet=None, accumulate: bool = False):
        """eq. 4 for one block.  Returns (y, logdet [B] float32 device tensor)."""
        import torch
        B = x.shape[0]
        y = torch.empty_like(x)
        if logdet is None:
            logdet = torch.zeros(B, dtype=torch.float32, device=x.device)
        _check(self.lib.sjd_forward_block(self._h, block, _dev(x, self._shape(B)), _dev(y), C.c_void_p(logdet.data_ptr()),
                                          1 if accumulate else 0, B, _stream_ptr()))
        return y, logdet

    def forward(self, x):
        """The whole forward map (blocks K-1 .. 0).  Returns (z, logdet [B])."""
        import torch
        B = x.shape[0]
        z = torch.empty_like(x)
        logdet = torch.zeros(B, dtype=torch.float32, device=x.device)
        _check(self.lib.sjd_forward(self._h, _dev(x, self._shape(B)), _dev(z), C.c_void_p(logdet.data_ptr()), B,
                                    _stream_ptr()))
        return z, logdet

    def sequential_inverse_block(self, block: int, z):
        import torch
        B = z.shape[0]
        x = torch.empty_like(z)
        _check(self.lib.sjd_sequential_inverse_block(self._h, block, _dev(z, self._shape(B)), _dev(x), B, _stream_ptr()))
        return x

    def sample(self, z, jacobi_mask: int, opts: JacobiOpts, out=None, want_iters: bool = True,
               allow_nonfinite: bool = False):
        """Returns (x, stats dict, iters int32 [K, B] or None)."""
        import torch
        B = z.shape[0]
        x = torch.empty_like(z) if out is None else out
        K = self.cfg.n_blocks
        stats = SjdStats()
        iters = np.zeros((K, B), np.int32) if want_iters else None
        ip = iters.ctypes.data_as(C.POINTER(C.c_int32)) if want_iters else None
        o = opts.c()
        _check(self.lib.sjd_sample(self._h, _dev(z, self._shape(B)), _dev(x, self._shape(B)), B,
                                   C.c_uint32(jacobi_mask & 0xFFFFFFFF), C.byref(o), C.byref(stats), ip, _stream_ptr()),
               allow_nonfinite)
        st = {"block_iters": list(stats.block_iters[:K]), "mean_sample_iters": list(stats.mean_sample_iters[:K]),
              "block_ms": list(stats.block_ms[:K])}
        return x, st, iters

    def set_mask_nearest(self, o: int) -> None:
        """Masked-dependency probe (eq. 6): attention ignores the o nearest preceding positions; 0 = off."""
        _check(self.lib.sjd_flow_set_mask_nearest(self._h, o))

    def set_sequential_path(self, path: int) -> None:
        """0 automatic, 1 per-step launches (graph replay), 2 persistent kernel, 3 the same with a plain launch."""
        _check(self.lib.sjd_flow_set_sequential_path(self._h, path))

    def set_projection_path(self, path: int) -> None:
        """0 automatic, 1 tile kernels + LayerNorm launches, 2 activation-stationary kernels (16-bit, width 512)."""
        _check(self.lib.sjd_flow_set_projection_path(self._h, path))

    def set_sequential_cus(self, n_cus: int) -> None:
        """Workgroups of the persistent sequential kernel: 0 = one per CU of the device, else a multiple of 32."""
        _check(self.lib.sjd_flow_set_sequential_cus(self._h, n_cus))

    def profile_enable(self, families) -> None:
        """Family indices (PROF_*); PROF_GEMM / PROF_DECODE_GEMM stand for every whole-sequence / single-token
        projection family."""
        mask = 0
        for f in families:
            mask |= 1 << f
            if f == PROF_GEMM:
                for g in PROF_GEMM_ALL:
                    mask |= 1 << g
            if f == PROF_DECODE_GEMM:
                for g in PROF_DECODE_GEMM_ALL:
                    mask |= 1 << g
        _check(self.lib.sjd_profile_enable(self._h, mask))

    def profile_read(self, reset: bool = True) -> dict:
        p = SjdProfile()
        _check(self.lib.sjd_profile_read(self._h, C.byref(p), 1 if reset else 0))
        out = {PROF_NAMES[i]: {"ms": p.ms[i], "launches": int(p.launches[i]), "flops": p.flops[i], "bytes": p.bytes[i]}
               for i in range(PROF_FAMILIES)}
        # all whole-sequence projections together, all single-token projections together
        out["gemm"] = {k: sum(out[PROF_NAMES[g]][k] for g in PROF_GEMM_ALL) for k in ("ms", "launches", "flops", "bytes")}
        out["decode_gemm"] = {k: sum(out[PROF_NAMES[g]][k] for g in PROF_DECODE_GEMM_ALL)
                              for k in ("ms", "launches", "flops", "bytes")}
        return out

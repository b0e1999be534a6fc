"""What the C entry points of the 4-bit cache and the head norms refuse, before any device is touched, and the plain format's own checks (CPU)."""
import ctypes as C

import numpy as np
import pytest

import paper_2505_24791_amd as sjd
from kv4_reference import LEVELS, held

PTR = 0x10000          # never followed: every call here is refused, or has nothing to do


@pytest.fixture(scope="module")
def lib():
    return sjd.load_library()


def _cache(**kw):
    d = dict(pages=PTR, n_pages=4, n_kv_heads=2, head_dim=64, dtype=sjd.DTYPE_F16)
    d.update(kw)
    return sjd.SjdKv4(*d.values())


def _opts(**kw):
    d = dict(norm=1, eps=1e-6, q_gain=None, q_shift=None, k_gain=None, k_shift=None, rot_dim=64, pairing=0, n_axes=2,
             axis_pairs=(C.c_int32 * 4)(16, 16, 0, 0), freq=PTR)
    d.update(kw)
    return sjd.SjdQkOpts(*d.values())


def _rope(lib, o, *, dtype=sjd.DTYPE_F16, pos=PTR, q=PTR, qs=256, heads=4, k=PTR, ks=128, kv=2, dim=64, qo=PTR, qos=256, ko=PTR, kos=128, n=3):
    return lib.sjd_op_qk_norm_rope(dtype, C.addressof(o) if o else None, pos, q, qs, heads, k, ks, kv, dim, qo, qos, ko, kos, n, None)


@pytest.mark.parametrize("o,kw,word", [
    (None, {}, "options"), ({}, dict(dtype=3), "dtype"), ({}, dict(dim=60), "head_dim"), ({}, dict(dim=264), "head_dim"),
    ({}, dict(n=-1), "n_rows"), ({}, dict(heads=0), "n_heads"), ({}, dict(q=None, k=None), "null"), ({}, dict(qo=None), "q_out_dev"),
    ({}, dict(q=PTR + 1), "element"), ({}, dict(qos=255), "stride"), ({}, dict(ks=-1), "stride"), ({}, dict(pos=None), "pos_dev"),
    (dict(norm=3), {}, "norm"), (dict(eps=-1.0), {}, "eps"), (dict(eps=float("nan")), {}, "eps"), (dict(norm=0, k_shift=PTR), {}, "norm"),
    (dict(rot_dim=72), {}, "rot_dim"), (dict(rot_dim=12), {}, "rot_dim"), (dict(pairing=2), {}, "pairing"), (dict(n_axes=0), {}, "n_axes"),
    (dict(n_axes=5), {}, "n_axes"), (dict(axis_pairs=(C.c_int32 * 4)(40, -8, 0, 0)), {}, "negative"),
    (dict(axis_pairs=(C.c_int32 * 4)(2 ** 31 - 1, 2 ** 31 - 1, 0, 0)), {}, "rot_dim / 2"), (dict(n_axes=1), {}, "rot_dim / 2"), (dict(freq=None), {}, "freq"),
    ({}, dict(n=2 ** 31 - 1, heads=65535), "too many")])
def test_norm_and_rotation_refuses(lib, o, kw, word):
    assert _rope(lib, _opts(**o) if o is not None else None, **kw) == sjd.SJD_EINVAL
    assert word in lib.sjd_last_error().decode()


@pytest.mark.parametrize("dim,rows", [(32, 2 ** 27), (64, 2 ** 26), (128, 2 ** 25), (256, 2 ** 24)])
def test_more_rows_than_a_launch_counts_are_refused(lib, dim, rows):
    c, w = _cache(head_dim=dim, n_kv_heads=4), 4 * dim
    calls = (lambda: lib.sjd_op_kv4_write(C.addressof(c), PTR, PTR, w, PTR, w, rows, None, None, None, 0, 0, None, 0, None),
             lambda: lib.sjd_op_kv4_read(C.addressof(c), PTR, PTR, w, PTR, w, rows, None),
             lambda: _rope(lib, _opts(norm=0, rot_dim=0, freq=None), heads=2, kv=2, dim=dim, qs=w, ks=w, qos=w, kos=w, n=rows))
    for call in calls:
        assert call() == sjd.SJD_EINVAL and "too many" in lib.sjd_last_error().decode()


def test_nothing_to_do_is_no_error(lib):
    assert _rope(lib, _opts(), n=0, q=None, k=None, qo=None, ko=None) == sjd.SJD_OK
    c = _cache(pages=None)
    assert lib.sjd_op_kv4_write(C.addressof(c), None, None, 0, None, 0, 0, None, None, None, 0, 0, None, 0, None) == sjd.SJD_OK
    assert lib.sjd_op_kv4_read(C.addressof(c), None, None, 0, None, 0, 0, None) == sjd.SJD_OK
    a = _attn(n_seqs=0, n_rows=0)
    assert lib.sjd_op_kv4_attention(C.addressof(c), C.addressof(a), None) == sjd.SJD_OK


@pytest.mark.parametrize("kw,word", [
    (dict(pages=None), "pages_dev"), (dict(pages=PTR + 8), "16-byte"), (dict(n_pages=0), "n_pages"), (dict(n_pages=2 ** 26), "n_pages"),
    (dict(n_kv_heads=0), "n_kv_heads"), (dict(head_dim=96), "head_dim"), (dict(head_dim=0), "head_dim"), (dict(dtype=7), "dtype")])
def test_caches_that_are_refused(lib, kw, word):
    c, a = _cache(**kw), _attn()
    calls = (lambda: lib.sjd_op_kv4_write(C.addressof(c), PTR, PTR, 128, PTR, 128, 3, None, None, None, 0, 0, None, 0, None),
             lambda: lib.sjd_op_kv4_read(C.addressof(c), PTR, PTR, 128, PTR, 128, 3, None),
             lambda: lib.sjd_op_kv4_attention(C.addressof(c), C.addressof(a), None))
    for call in calls:
        assert call() == sjd.SJD_EINVAL and word in lib.sjd_last_error().decode()


@pytest.mark.parametrize("at,value,word", [
    (0, None, "slot_dev"), (1, None, "k_dev"), (1, PTR + 1, "k_dev"), (2, -1, "k_dev"), (3, None, "v_dev"), (5, -3, "n_rows"), (8, PTR, "opts")])
def test_writes_that_are_refused(lib, at, value, word):
    c = _cache()
    args = [PTR, PTR, 128, PTR, 128, 3, None, None, None, 256, 4, PTR, 256]
    args[at] = value
    assert lib.sjd_op_kv4_write(C.addressof(c), *args, None) == sjd.SJD_EINVAL and word in lib.sjd_last_error().decode()


def test_fused_writes_that_are_refused(lib):
    o = _opts()
    for c, heads, qo, word in ((_cache(n_kv_heads=200), 400, PTR, "8192"), (_cache(), 3, PTR, "multiple"), (_cache(), 4, None, "q_out_dev")):
        assert lib.sjd_op_kv4_write(C.addressof(c), PTR, PTR, 1 << 15, PTR, 1 << 15, 3, C.addressof(o), PTR, PTR, 1 << 15, heads, qo, 1 << 15, None) == sjd.SJD_EINVAL
        assert word in lib.sjd_last_error().decode()


def test_reads_that_are_refused(lib):
    c = _cache()
    for args, word in (((None, PTR, 128, PTR, 128, 3), "slot_dev"), ((PTR, None, 128, PTR, 128, 3), "k_dev"), ((PTR, PTR, 127, PTR, 128, 3), "stride"),
                       ((PTR, PTR, 128, PTR + 1, 128, 3), "v_dev"), ((PTR, PTR, 128, PTR, 128, -1), "n_rows")):
        assert lib.sjd_op_kv4_read(C.addressof(c), *args, None) == sjd.SJD_EINVAL and word in lib.sjd_last_error().decode()


def _attn(**kw):
    d = dict(q=PTR, o=PTR, q_stride=256, o_stride=256, table_stride=4, q_start=None, kv_len=PTR, page_table=PTR, n_seqs=3, n_heads=4, n_rows=3,
             max_pages=4, max_q=1, max_kv=256, causal=1, skip_nearest=0, window=0, scale=0.125, workspace=None, workspace_bytes=0)
    d.update(kw)
    return sjd.SjdKv4Attention(*d.values())


@pytest.mark.parametrize("kw,word", [
    (dict(q=None), "q_dev"), (dict(o=None), "o_dev"), (dict(o=PTR + 1), "o_dev"), (dict(o_stride=255), "stride"), (dict(q_stride=-1), "stride"),
    (dict(kv_len=None), "kv_len_dev"), (dict(page_table=None), "page_table"), (dict(table_stride=-1), "table_stride"), (dict(n_heads=3), "multiple"),
    (dict(n_heads=0), "multiple"), (dict(n_seqs=-1), "negative"), (dict(max_q=-1), "negative"), (dict(max_kv=-1), "negative"), (dict(max_pages=-1), "negative"),
    (dict(n_rows=4), "max_q rows"), (dict(skip_nearest=-1), "skip_nearest"), (dict(window=-1), "window"), (dict(scale=0.0), "scale"),
    (dict(scale=float("inf")), "scale"), (dict(scale=float("nan")), "scale"), (dict(max_kv=2 ** 31 - 1), "out of range"),
    (dict(max_pages=2 ** 26), "out of range")])
def test_attention_that_is_refused(lib, kw, word):
    c, a = _cache(), _attn(**kw)
    assert lib.sjd_op_kv4_attention(C.addressof(c), C.addressof(a), None) == sjd.SJD_EINVAL
    assert word in lib.sjd_last_error().decode()


@pytest.mark.parametrize("kw,word", [
    (dict(scale=3e38), "scale"), (dict(scale=float("nan")), "scale"), (dict(scale=float("inf")), "scale"), (dict(n_seqs=65536, n_rows=65536), "too many"),
    (dict(n_heads=64, max_q=2 ** 21, n_rows=3 * 2 ** 21), "too many")])
def test_attention_beyond_its_ranges_is_refused(lib, kw, word):
    a, c, n = _attn(**kw), _cache(), C.c_size_t()
    for call in (lambda: lib.sjd_op_kv4_attention(C.addressof(c), C.addressof(a), None),
                 lambda: lib.sjd_kv4_attention_workspace(C.addressof(c), C.addressof(a), C.addressof(n))):
        assert call() == sjd.SJD_EINVAL and word in lib.sjd_last_error().decode()


def test_attention_asks_for_its_workspace(lib):
    c, need = _cache(), C.c_size_t(0)
    a = _attn(max_pages=4000, max_kv=250000)
    assert lib.sjd_kv4_attention_workspace(C.addressof(c), C.addressof(a), C.addressof(need)) == sjd.SJD_OK and need.value > 0
    for ws, n in ((None, 0), (PTR, need.value - 1), (PTR + 4, need.value)):
        a.workspace, a.workspace_bytes = ws, n
        assert lib.sjd_op_kv4_attention(C.addressof(c), C.addressof(a), None) == sjd.SJD_EINVAL
        assert str(need.value) in lib.sjd_last_error().decode()
    short = _attn()
    assert lib.sjd_kv4_attention_workspace(C.addressof(c), C.addressof(short), C.addressof(need)) == sjd.SJD_OK and need.value == 0
    assert lib.sjd_kv4_attention_workspace(C.addressof(c), C.addressof(short), None) == sjd.SJD_EINVAL


def test_reference_format():
    """The plain form that the GPU tests hold the kernels to: every value by trying all levels."""
    rng = np.random.default_rng(0)
    x = rng.standard_normal((50, 64)) * 2.0 ** rng.integers(-20, 12, (50, 1))
    got = held(x, "bfloat16").reshape(50, 2, 32)
    g = x.reshape(50, 2, 32)
    for i in range(50):
        for j in range(2):
            e = next(e for e in range(-125, 126) if np.abs(g[i, j]).max() <= 7 * 2.0 ** e)
            every = np.concatenate([-LEVELS[::-1], LEVELS]) * 2.0 ** e
            want = every[np.abs(g[i, j][:, None] - every).argmin(1)]
            assert np.array_equal(got[i, j], want)
    assert np.array_equal(held(np.array([[0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.5, 7.0, -0.25, -5.0] + [0.0] * 21]), "float32")[0, :11],
                          [0, 1, 1, 2, 2, 4, 4, 6, 6, 0, -4])

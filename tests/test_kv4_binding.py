"""What the binding of the head norms and the 4-bit cache refuses before the library is called: a stub stands in for the library (CPU)."""
import contextlib

import pytest
import torch

import paper_2505_24791_amd as sjd


class Stub:
    """Entry points that only write down what they were called with."""

    def __init__(self):
        self.calls = []

    def __getattr__(self, name):
        return lambda *args: self.calls.append((name, args)) or 0


@pytest.fixture
def stub(monkeypatch):
    lib = Stub()
    types = {torch.float16: sjd.DTYPE_F16, torch.bfloat16: sjd.DTYPE_BF16, torch.float32: sjd.DTYPE_F32}
    monkeypatch.setattr(sjd, "_rt", (lib, lambda device: 0, lambda: 0, lambda device: contextlib.nullcontext(), torch.int32, types))
    return lib


@pytest.mark.parametrize("norm", ["none", "rms", "layer"])
@pytest.mark.parametrize("side", ["q", "k", "both"])
def test_rows_in_host_memory_are_refused(stub, norm, side):
    """Options without vectors belong to no device: nothing but the rows says where they are."""
    x = torch.zeros((4, 2, 64), dtype=torch.float16)
    q, k = (x if side != "k" else None), (x if side != "q" else None)
    with pytest.raises(sjd.SjdError, match="GPU"):
        sjd.op_qk_norm_rope(q, k, None, sjd.QkOpts(norm=norm))
    with pytest.raises(sjd.SjdError):
        sjd.op_qk_norm_rope(q, k, None, sjd.QkOpts(norm=norm), q_out=q, k_out=k)
    assert not stub.calls


class Fake:
    """What the binding looks at of a tensor on the GPU."""
    is_cuda = True

    def __init__(self, shape, dtype, at=0x10000, stride=None, device=0):
        self.shape, self.dtype, self.at, self.device = torch.Size(shape), dtype, at, device
        steps = [1]
        for n in reversed(shape[1:]):
            steps.insert(0, steps[0] * n)
        self.steps = tuple(stride or steps)

    def stride(self):
        return self.steps

    def get_device(self):
        return self.device

    def data_ptr(self):
        return self.at

    def dim(self):
        return len(self.shape)

    def numel(self):
        return self.shape.numel()

    def is_contiguous(self):
        return True

    def new_empty(self, shape, dtype=None):
        return Fake(shape, dtype or self.dtype, 0x900000)


def _struct(address, kind):
    return kind.from_address(address)


def test_options_follow_their_tensors(stub):
    """A gain or a table of frequencies whose storage is replaced (``param.data = ...``, a module that moves) is read where it is now."""
    gain, freq, x = Fake((64,), torch.float32, 0x1000), Fake((32,), torch.float32, 0x2000), Fake((4, 2, 64), torch.float16)
    o = sjd.QkOpts(q_gain=gain, freq=freq, rot_dim=64, axis_pairs=(32,))
    pos = Fake((4, 1), torch.int32)
    seen = lambda: (lambda c: (c.q_gain, c.freq))(_struct(stub.calls[-1][1][1], sjd.SjdQkOpts))
    sjd.op_qk_norm_rope(x, None, pos, o)
    assert seen() == (0x1000, 0x2000)
    gain.at = 0x3000
    sjd.op_qk_norm_rope(x, None, pos, o)
    assert seen() == (0x3000, 0x2000)
    freq.at = 0x4000
    cache = sjd.Kv4Cache(Fake((2, 2, 68 * 64), torch.uint8), torch.float16)
    sjd.op_kv4_write(cache, x, x, Fake((4,), torch.int32), opts=o, pos=pos)
    assert _struct(stub.calls[-1][1][7], sjd.SjdQkOpts).freq == 0x4000
    done = len(stub.calls)
    for t, change, back in ((gain, dict(at=0), dict(at=0x3000)),                                # freed: a null gain would be taken for ones
                            (gain, dict(at=0x5000, dtype=torch.float16), dict(at=0x3000, dtype=torch.float32)),
                            (gain, dict(at=0x5000, is_cuda=False, device=-1), dict(at=0x3000, is_cuda=True, device=0)),
                            (freq, dict(at=0x5000, shape=torch.Size((16,))), dict(at=0x4000, shape=torch.Size((32,))))):
        vars(t).update(change)
        for _ in range(2):                                                                      # and again, not the first time alone
            with pytest.raises(sjd.SjdError):
                sjd.op_qk_norm_rope(x, None, pos, o)
        vars(t).update(back)
        assert len(stub.calls) == done
    sjd.op_qk_norm_rope(x, None, pos, o)
    assert seen() == (0x3000, 0x4000)


def test_caches_follow_their_pages(stub):
    pages = Fake((2, 2, 68 * 64), torch.uint8, 0x1000)
    cache = sjd.Kv4Cache(pages, torch.float16)
    x, i32 = Fake((4, 2, 64), torch.float16), lambda *s: Fake(s, torch.int32)
    calls = (lambda: sjd.op_kv4_write(cache, x, x, i32(4)), lambda: sjd.op_kv4_read(cache, i32(4)),
             lambda: sjd.op_kv4_attention(cache, x, i32(4, 1), i32(4)))
    for i, call in enumerate(calls):
        pages.at = 0x2000 + 0x100 * i
        call()
        assert _struct(stub.calls[-1][1][0], sjd.SjdKv4).pages == pages.at
    cache.pages = Fake((7, 2, 68 * 64), torch.uint8, 0x8000)                                     # a larger cache in its place
    calls[0]()
    c = _struct(stub.calls[-1][1][0], sjd.SjdKv4)
    assert (c.pages, c.n_pages) == (0x8000, 7) and cache.n_pages == 7
    done = len(stub.calls)
    cache.pages = Fake((7, 2, 68 * 64), torch.int8, 0x9000)
    for call in calls * 2:
        with pytest.raises(sjd.SjdError):
            call()
    assert len(stub.calls) == done


MANY = 2 ** 32 + 4          # 4 to a call that counts in 32 bits


def test_counts_beyond_32_bits_are_refused(stub):
    """Rows that all lie in the same memory (``expand``) can be so many, and so can a page table's entries."""
    i32 = lambda *s: Fake(s, torch.int32)
    rows = lambda n, h, d: Fake((n, h, d), torch.float16, stride=(0 if n == MANY else h * d, d, 1))
    cache = sjd.Kv4Cache(Fake((2, 2, 68 * 64), torch.uint8), torch.float16)
    none, x = sjd.QkOpts(), rows(4, 2, 64)
    for call in (lambda: sjd.op_qk_norm_rope(rows(MANY, 2, 64), None, None, none), lambda: sjd.op_qk_norm_rope(None, rows(MANY, 2, 64), None, none),
                 lambda: sjd.op_qk_norm_rope(rows(4, MANY, 64), None, None, none), lambda: sjd.op_qk_norm_rope(rows(4, 1, MANY + 60), None, None, none),
                 lambda: sjd.op_kv4_write(cache, rows(MANY, 2, 64), rows(MANY, 2, 64), i32(MANY)),
                 lambda: sjd.op_kv4_write(cache, x, x, i32(4), q=rows(4, MANY, 64), opts=none),
                 lambda: sjd.op_kv4_read(cache, i32(MANY)),
                 lambda: sjd.op_kv4_attention(cache, rows(MANY, 2, 64), i32(MANY, 1), i32(MANY)),
                 lambda: sjd.op_kv4_attention(cache, rows(4, MANY, 64), i32(4, 1), i32(4)),
                 lambda: sjd.op_kv4_attention(cache, x, i32(MANY, 1), i32(MANY), q_start=i32(MANY + 1)),
                 lambda: sjd.op_kv4_attention(cache, x, i32(4, MANY), i32(4), max_kv=100),
                 lambda: sjd.QkOpts(rot_dim=64, axis_pairs=(2 ** 32 + 16, 16), freq=Fake((32,), torch.float32)),
                 lambda: sjd.QkOpts(rot_dim=64, axis_pairs=(2 ** 32 + 16, 16 - 2 ** 32), freq=Fake((32,), torch.float32))):
        with pytest.raises(sjd.SjdError):
            call()
    assert not stub.calls


def test_a_rotation_without_positions_is_refused(stub):
    o = sjd.QkOpts(rot_dim=64, axis_pairs=(32,), freq=Fake((32,), torch.float32))
    x, cache = Fake((4, 2, 64), torch.float16), sjd.Kv4Cache(Fake((2, 2, 68 * 64), torch.uint8), torch.float16)
    for call in (lambda: sjd.op_qk_norm_rope(x, None, None, o), lambda: sjd.op_kv4_write(cache, x, x, Fake((4,), torch.int32), opts=o)):
        with pytest.raises(sjd.SjdError, match="pos"):
            call()
    assert not stub.calls

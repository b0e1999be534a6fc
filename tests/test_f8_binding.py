"""What the binding of the 8-bit rows refuses, and what it hands to the library: a stub stands in for the library (CPU)."""
import contextlib
import struct

import pytest
import torch

import paper_2505_24791_amd as sjd
from test_kv4_binding import Fake, Stub

U8, F8, F16, BF16, F32 = torch.uint8, torch.float8_e4m3fn, torch.float16, torch.bfloat16, torch.float32


@pytest.fixture
def stub(monkeypatch):
    lib = Stub()
    types = {F16: sjd.DTYPE_F16, BF16: sjd.DTYPE_BF16, F32: sjd.DTYPE_F32}
    monkeypatch.setattr(sjd, "_rt", (lib, lambda device: 0, lambda: 0, lambda device: contextlib.nullcontext(), torch.int32, types, U8, F8, F16))
    return lib


def _fake(shape, dtype, at=0x10000, **kw):
    if isinstance(shape, int):
        shape = (shape,)
    return Fake(shape, dtype, at, **kw)


class Alloc(Fake):
    def new_empty(self, shape, dtype=None):
        return Alloc((shape,) if isinstance(shape, int) else shape, dtype or self.dtype, 0x900000)


def _rows(n=3, width=200, **kw):
    groups = -(-width // 128)
    return sjd.F8Rows(Alloc((n, groups * 128), kw.get("dtype", U8), kw.get("at", 0x10000), device=kw.get("device", 0)),
                      Alloc((n, (groups + 3) // 4 * 4), U8, kw.get("s_at", 0x20000), device=kw.get("s_device", kw.get("device", 0))), width)


def _struct(packed):
    return struct.unpack("PPqqii", packed)


def test_rows_are_what_their_tensors_are_then(stub):
    r = _rows()
    assert _struct(r._now("rows")) == (0x10000, 0x20000, 256, 4, 3, 200) and r.n_rows == 3 and r.device == 0
    r.codes.at = 0x30000                                             # a storage that was replaced
    assert _struct(r._now("rows"))[0] == 0x30000
    r.scales = Alloc((3, 4), U8, 0x40000, stride=(8, 1))
    assert _struct(r._now("rows")) == (0x30000, 0x40000, 256, 8, 3, 200)
    r.codes = Alloc((3, 256), F8, 0x50000, stride=(512, 1))
    assert _struct(r._now("rows")) == (0x50000, 0x40000, 512, 8, 3, 200)
    one = sjd.F8Rows(Alloc((1, 256), U8, stride=(7, 1)), Alloc((1, 4), U8, stride=(3, 1)), 200)     # a single row has no next one
    assert _struct(one._now("rows"))[2:] == (256, 4, 1, 200)


def test_rows_made_by_a_call_follow_their_memory(stub):
    """Both parts are in one allocation; whoever asks gets tensors of them, and a copy of the object is its own."""
    import copy
    x = torch.zeros(3, 200)
    x.get_device = lambda: 0
    r = sjd.F8Rows.empty(3, 200, x)
    at = r._both.data_ptr()
    assert _struct(r._now("rows")) == (at, at + 3 * 256, 256, 4, 3, 200)
    other = copy.deepcopy(r)
    r.codes.fill_(1)
    assert r.codes.shape == (3, 256) and r.scales.shape == (3, 4) and r.codes.data_ptr() == at and r.scales.data_ptr() == at + 3 * 256
    assert other.codes.data_ptr() != at and not torch.equal(other.codes, torch.ones_like(other.codes))
    with pytest.raises(sjd.SjdError, match="GPU"):                       # both copies lie in host memory, in truth
        r._now("rows")
    with pytest.raises(sjd.SjdError, match="GPU"):
        other._now("rows")
    none = sjd.F8Rows.empty(0, 200, x)
    assert none.codes.shape == (0, 256) and none.scales.shape == (0, 4)
    for n, width, like in ((3, 0, x), (3, (1 << 20) + 1, x), (2 ** 31, 200, x), (3, 200, torch.zeros(1))):
        with pytest.raises(sjd.SjdError):
            sjd.F8Rows.empty(n, width, like)


def test_rows_that_threads_share(stub):
    """A weight that one thread hands to calls while another asks for its tensors: every call gets the struct of its memory, or finds it on the host."""
    import sys
    import threading
    x = torch.zeros(1, 1)
    x.get_device = lambda: 0
    went, before = [], sys.getswitchinterval()
    sys.setswitchinterval(1e-6)
    try:
        for _ in range(200):
            r = sjd.F8Rows.empty(3, 200, x)
            at, start = r._both.data_ptr(), threading.Barrier(4)
            whole = (at, at + 3 * 256, 256, 4, 3, 200)

            def call():
                start.wait()
                for _ in range(5):
                    try:
                        went.append(_struct(r._now("rows")) == whole and r._like().data_ptr() == at)
                    except sjd.SjdError as e:
                        went.append("GPU" in str(e))
                    except Exception as e:
                        went.append(e)

            def ask():
                start.wait()
                try:
                    went.append(r.codes.data_ptr() == at and r.scales.data_ptr() == at + 3 * 256)
                except Exception as e:
                    went.append(e)

            threads = [threading.Thread(target=f) for f in (call, call, ask, ask)]
            for th in threads:
                th.start()
            for th in threads:
                th.join()
    finally:
        sys.setswitchinterval(before)
    assert len(went) == 200 * 12 and all(w is True for w in went)


@pytest.mark.parametrize("codes,scales,width,word", [
    (((3, 256), F16), ((3, 4), U8), 200, "codes"), (((3, 255), U8), ((3, 4), U8), 200, "codes"), (((3, 384), U8), ((3, 4), U8), 200, "codes"), (((3, 2, 128), U8), ((3, 4), U8), 200, "codes"),
    (((3, 256), U8), ((3, 2), U8), 200, "scales"), (((3, 256), U8), ((4, 4), U8), 200, "scales"), (((3, 256), U8), ((3, 4), F32), 200, "scales"),
    (((3, 256), U8), ((3, 4), U8), 0, "width"), (((3, 256), U8), ((3, 4), U8), 200.0, "width"), (((3, 256), U8), ((3, 4), U8), True, "width"), (((3, 256), U8), ((3, 4), U8), (1 << 20) + 1, "width"),
    (((2 ** 31, 256), U8), ((2 ** 31, 4), U8), 200, "too many")])
def test_rows_of_another_form_are_refused(stub, codes, scales, width, word):
    with pytest.raises(sjd.SjdError, match=word):
        sjd.op_f8_read(sjd.F8Rows(Alloc(*codes), Alloc(*scales), width), F16)
    assert not stub.calls


def test_strides_and_devices_of_rows(stub):
    for r in (sjd.F8Rows(Alloc((3, 256), U8, stride=(512, 2)), Alloc((3, 4), U8), 200), sjd.F8Rows(Alloc((3, 256), U8), Alloc((3, 4), U8, stride=(8, 2)), 200),
              _rows(s_device=1), _rows(device=-1)):
        with pytest.raises(sjd.SjdError):
            sjd.op_f8_read(r, F16)
    with pytest.raises(sjd.SjdError, match="one GPU"):
        sjd.op_linear_f8(_rows(), _rows(5, device=1))
    with pytest.raises(sjd.SjdError, match="one GPU"):
        sjd.op_gated_mlp_f8(_rows(), _rows(12), _rows(7, 6, device=1))
    assert not stub.calls


X = dict(x=((3, 200), F16))


@pytest.mark.parametrize("kw,word", [
    (dict(x=((3, 200), torch.float64)), "float16"), (dict(x=((3, 200), F16, dict(device=-1))), "GPU"), (dict(x=((3, 2, 100), F16)), "rows"), (dict(x=((3, 200), F16, dict(stride=(400, 2)))), "following"),
    (dict(norm="batch"), "norm"), (dict(gain=((199,), F32)), "gain"), (dict(gain=((200,), F16)), "gain"), (dict(shift=((200,), F32, dict(device=1))), "shift"),
    (dict(resid=((3, 199), F32)), "resid"), (dict(resid=((3, 200), torch.float64)), "float16"), (dict(resid=((3, 200), F32, dict(device=1))), "resid"), (dict(x=((3, 0), F16)), "values"),
    (dict(x=((3, (1 << 20) + 1), F16)), "values"), (dict(x=((2 ** 31, 200), F16)), "too many")])
def test_norm_refuses(stub, kw, word):
    made = {k: Alloc(*v[:2], **(v[2] if len(v) > 2 else {})) if isinstance(v, tuple) else v for k, v in {**X, **kw}.items()}
    with pytest.raises(sjd.SjdError, match=word):
        sjd.op_norm_f8(made.pop("x"), **made)
    assert not stub.calls


def test_norm_hands_over_what_it_was_given(stub):
    x = Alloc((3, 200), BF16, 0x1000, stride=(300, 1))
    out = sjd.op_norm_f8(x, resid=Alloc((3, 200), F32, 0x2000, stride=(256, 1)), norm="layer", gain=Alloc((200,), F32, 0x3000), shift=Alloc((200,), F32, 0x4000), eps=1e-5)
    (name, args), = stub.calls
    assert name == "sjd_op_norm_f8" and args[:10] == (sjd.DTYPE_BF16, 0x1000, 300, sjd.DTYPE_F32, 0x2000, 256, 2, 1e-5, 0x3000, 0x4000)
    assert _struct(args[10]) == (0x900000, 0x900000 + 3 * 256, 256, 4, 3, 200) and out.n_rows == 3 and out.width == 200
    stub.calls.clear()
    given = _rows()
    assert sjd.op_norm_f8(x, norm="none", out=given) is given
    assert stub.calls[0][1][3:10] == (sjd.DTYPE_BF16, None, 0, 0, 1e-6, None, None)
    for other in (_rows(4), _rows(width=201), _rows(device=1)):
        with pytest.raises(sjd.SjdError, match="out"):
            sjd.op_norm_f8(x, out=other)


@pytest.mark.parametrize("kw,word", [
    (dict(bias=((4,), F32)), "bias"), (dict(bias=((5,), F16)), "bias"), (dict(dtype=torch.float64), "float16"), (dict(out=((3, 6), F16)), "shape"), (dict(out=((3, 5), F16), dtype=BF16), "out"),
    (dict(out=((3, 5), torch.int32)), "float16"), (dict(resid=((3, 5), F16)), "float32"), (dict(resid=((3, 5), F32), dtype=F16), "float32"), (dict(resid=((3, 5), F32), out=((3, 5), F32)), "resid"),
    (dict(resid=((3, 6), F32)), "shape"), (dict(out=((3, 5), F16, dict(device=1))), "out"), (dict(out=((3, 5), F16, dict(stride=(10, 2)))), "following")])
def test_projections_refuse(stub, kw, word):
    make = lambda: {k: Alloc(*v[:2], **(v[2] if len(v) > 2 else {})) if isinstance(v, tuple) else v for k, v in kw.items()}  # noqa: E731
    with pytest.raises(sjd.SjdError, match=word):
        sjd.op_linear_f8(_rows(), _rows(5), **make())
    if "bias" not in kw:
        with pytest.raises(sjd.SjdError, match=word):
            sjd.op_gated_mlp_f8(_rows(), _rows(12), _rows(5, 6), **make())
    assert all(name.endswith("workspace") for name, _ in stub.calls)
    with pytest.raises(sjd.SjdError, match="activation"):
        sjd.op_gated_mlp_f8(_rows(), _rows(12), _rows(5, 6), activation="relu")


def test_projections_hand_over_what_they_were_given(stub):
    x, w = _rows(), _rows(5, at=0x50000, s_at=0x60000)
    out = sjd.op_linear_f8(x, w, bias=Alloc((5,), F32, 0x7000))
    name, args = stub.calls[-1]
    assert name == "sjd_op_linear_f8" and out.dtype is F16 and tuple(out.shape) == (3, 5)
    assert _struct(args[0])[:2] == (0x10000, 0x20000) and _struct(args[1])[:2] == (0x50000, 0x60000) and args[2:7] == (0x7000, sjd.DTYPE_F16, 0x900000, 5, 0)
    assert sjd.op_linear_f8(x, w, dtype=BF16).dtype is BF16 and sjd.op_linear_f8(x, w, dtype=F32).dtype is F32
    r = Alloc((3, 5), F32, 0x8000, stride=(9, 1))
    assert sjd.op_linear_f8(x, w, resid=r) is r and stub.calls[-1][1][2:7] == (None, sjd.DTYPE_F32, 0x8000, 9, 1)
    o = Alloc((3, 5), BF16, 0x9000, stride=(6, 1))
    assert sjd.op_linear_f8(x, w, out=o) is o and stub.calls[-1][1][3:7] == (sjd.DTYPE_BF16, 0x9000, 6, 0)
    assert sjd.op_gated_mlp_f8(x, _rows(12), _rows(5, 6), activation="gelu", resid=r) is r
    assert stub.calls[-2][0] == "sjd_gated_mlp_f8_workspace" and stub.calls[-2][1][2] == sjd.DTYPE_F32
    assert stub.calls[-1][1][3:8] == (1, sjd.DTYPE_F32, 0x8000, 9, 1)


def test_rows_whose_form_changes_in_place(stub):
    """The tensors of the same addresses with other rows, strides or types: resized, or given another tensor's data that begins at the same place."""
    r = _rows(50)
    assert _struct(r._now("rows")) == (0x10000, 0x20000, 256, 4, 50, 200)
    r.codes.shape, r.scales.shape = torch.Size((10, 256)), torch.Size((10, 4))
    assert _struct(r._now("rows")) == (0x10000, 0x20000, 256, 4, 10, 200)
    r.codes.steps, r.scales.steps = (512, 1), (8, 1)
    assert _struct(r._now("rows")) == (0x10000, 0x20000, 512, 8, 10, 200)
    with pytest.raises(sjd.SjdError, match="out"):
        sjd.op_norm_f8(Alloc((50, 200), F16), out=r)
    for change, back in ((dict(shape=torch.Size((10, 384))), dict(shape=torch.Size((10, 256)))), (dict(dtype=F16), dict(dtype=U8)), (dict(steps=(512, 2)), dict(steps=(512, 1))),
                         (dict(device=1), dict(device=0))):
        for name, value in change.items():
            setattr(r.codes, name, value)
        with pytest.raises(sjd.SjdError):
            r._now("rows")
        for name, value in back.items():
            setattr(r.codes, name, value)
        assert _struct(r._now("rows")) == (0x10000, 0x20000, 512, 8, 10, 200)
    assert not stub.calls


def test_a_call_sees_one_form_of_rows_that_another_thread_replaces(stub, monkeypatch):
    """The struct, the device and the number of rows that a call goes by are of one look: another thread replaces the tensors and looks at them in the middle of it."""
    class There(Alloc):
        def new_empty(self, shape, dtype=None):
            return There((shape,) if isinstance(shape, int) else shape, dtype or self.dtype, 0x900000, device=self.device)

    pack = sjd._SJD_F8
    r = _rows(9)

    def while_another_thread_replaces(*values):
        if values[4] == 9:
            monkeypatch.setattr(sjd, "_SJD_F8", pack)
            r.codes, r.scales = There((3, 256), U8, 0x70000, device=1), There((3, 4), U8, 0x80000, device=1)
            assert _struct(r._now("rows")) == (0x70000, 0x80000, 256, 4, 3, 200)
        return pack(*values)

    def start():
        r.codes, r.scales = There((9, 256), U8), There((9, 4), U8, 0x20000)
        monkeypatch.setattr(sjd, "_SJD_F8", while_another_thread_replaces)

    for call, shape in ((lambda: sjd.op_f8_read(r, F16), (9, 200)), (lambda: sjd.op_linear_f8(r, _rows(5)), (9, 5)), (lambda: sjd.op_linear_f8(r, _rows(5), out=Alloc((9, 5), F16)), (9, 5)),
                        (lambda: sjd.op_linear_f8(_rows(2), r), (2, 9)), (lambda: sjd.op_gated_mlp_f8(r, _rows(12), _rows(5, 6)), (9, 5))):
        start()
        out = call()
        assert tuple(out.shape) == shape and out.device == 0
    start()
    assert sjd.op_norm_f8(Alloc((9, 200), F16), out=r) is r and _struct(stub.calls[-1][1][10])[4] == 9


def test_rows_say_how_many_they_are_and_where_before_any_call(stub):
    r = _rows(5, device=1)
    assert r.n_rows == 5 and r.device == 1
    r.codes, r.scales = Alloc((7, 256), U8), Alloc((7, 4), U8)
    assert r.n_rows == 7 and r.device == 0
    x = torch.zeros(3, 200)
    x.get_device = lambda: 0
    made = sjd.F8Rows.empty(3, 200, x)
    assert made.n_rows == 3 and made.device == 0
    made.codes = Alloc((9, 256), U8, device=2)
    assert made.n_rows == 9 and made.device == 2


def test_tensors_set_while_another_thread_asks_for_the_made_ones_stay(stub):
    """Making tensors of the parts takes a while; what another thread sets meanwhile is not lost, and all who ask get the same tensors."""
    import threading
    for use in ("set", "ask"):
        inside, go_on, went = threading.Event(), threading.Event(), []

        class Slow(torch.Tensor):
            def split(self, sizes):
                first, inside_before = not inside.is_set(), inside.set()
                if first:
                    go_on.wait(0.5)
                return torch.Tensor.split(self, sizes)

        x = torch.zeros(3, 200)
        x.get_device = lambda: 0
        r = sjd.F8Rows.empty(3, 200, x)
        r._both = r._both.as_subclass(Slow)
        mine = Alloc((3, 256), U8, 0x70000)

        def second():
            inside.wait(5)
            if use == "set":
                r.codes = mine
            went.append(r.codes)
            go_on.set()

        one, two = threading.Thread(target=lambda: went.append(r.scales)), threading.Thread(target=second)
        one.start(), two.start(), one.join(), two.join()
        assert len(went) == 2
        if use == "set":
            assert r.codes is mine
        else:
            assert any(t is r.codes for t in went) and any(t is r.scales for t in went)

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

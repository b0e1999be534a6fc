"""The gated block of 8-bit rows where its hidden values are easily wrong: gates in the tail of the activation, results of three more bits than
bfloat16's, results added to the stream; projections into the stream by every tile.

Tolerances.  Hidden values lie on a grid of 8-bit floats: half a step, 2^-4 of a value or 2^-10 of a scale (at least the group's largest / 448).  The activation's float32 arithmetic
is off by what the exponent of 2 is rounded by, 2^-24 of it twice and 2^-25 for its constant (it is at most 116 for the gates here: 2.5 * 116 * 2^-24 ln 2 < 2^-16), and by less than 2^-18 for the rest.
Sums of integers are exact.
"""
import math

import pytest
import torch

import f8_reference as ref
import paper_2505_24791_amd as sjd
from test_gpu_f8 import BF16, F16, F32, TYPES, _gen, _integers_gpu, _rows

pytestmark = pytest.mark.gpu

# rows, width, hidden channels: each launch that the gate has (few rows, few rows with long k, tiles, and tiles that fill the chip)
LAUNCHES = [(5, 200, 256), (40, 1100, 640), (400, 1100, 1280), (3000, 300, 640), (9000, 300, 2304)]


def _picked(hidden, n, g):
    """A weight that picks n hidden channels, so that what is held is seen as it is."""
    pick = torch.randint(0, hidden, (n,), generator=g)
    w = torch.zeros(n, hidden)
    w[torch.arange(n), pick] = 1
    return pick, _rows(*ref.hold(w), hidden)


@pytest.mark.parametrize("m,width,hidden", LAUNCHES)
@pytest.mark.parametrize("act,low,high", [("gelu", -8.0, -4.0), ("gelu", -12.0, -8.0), ("gelu", -4.0, 4.0), ("silu", -16.0, -8.0), ("silu", -80.0, -64.0), ("silu", -4.0, 4.0)])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_a_group_of_gates_in_the_tail_keeps_its_bits(m, width, hidden, act, low, high, dtype):
    """All gates of 128 channels lie between `low` and `high`: their hidden values are held by a scale of their own, so each has to be right relative to itself."""
    g = _gen(hidden)
    # a row is (1, 2^-4, zeros): a gate is a + b / 16 with two values of the grid, exactly
    x = torch.zeros(m, width)
    x[:, 0], x[:, 1] = 1.0, 0.0625
    step = (high - low) / 16
    gate = torch.zeros(hidden, width)
    gate[:, 0] = low + step * torch.randint(0, 16, (hidden,), generator=g)
    gate[:, 1] = step * torch.randint(0, 15, (hidden,), generator=g)
    gate = ref.values(*ref.hold(gate), width).float()                      # as the grid has them
    up = torch.zeros(hidden, width)
    up[:, 0] = 1.0
    z = (x[:1].double() @ gate.double().T)[0]
    assert float(z.min()) >= low - abs(low) / 16 and float(z.max()) <= high + abs(high) / 8 + 1
    h = ref.activation(z, act)
    top = torch.nn.functional.pad(h.abs(), (0, -hidden % 128)).view(-1, 128).amax(-1)
    grid = 2.0 ** -10 * torch.repeat_interleave(torch.exp2(torch.ceil(torch.log2(top * (1 + 2.0 ** -16) / 448))), 128)[:hidden]
    near = h.abs() * (2.0 ** -16 + 2.0 ** -18)
    far = near + torch.maximum((h.abs() + near) * 2.0 ** -4, grid)
    pick, w_out = _picked(hidden, 100, g)
    got = sjd.op_gated_mlp_f8(_rows(*ref.hold(x), width), _rows(*ref.hold(torch.cat((gate, up))), width), w_out, activation=act, dtype=dtype).cpu().double()
    assert torch.equal(got, got[:1].expand_as(got))
    want, far = h[pick], far[pick]
    far = far if dtype is F32 else far + torch.finfo(dtype).eps / 2 * (want.abs() + far)
    off = (got[0] - want).abs() / far
    assert float(off.max()) <= 1, (float(off.max()), float(z[pick][off.argmax()]))


@pytest.mark.parametrize("m,width,hidden", LAUNCHES + [(16400, 512, 1408), (9100, 520, 2307)])
@pytest.mark.parametrize("act", ["silu", "gelu"])
def test_half_results_are_as_near_as_float32_sums_make_them(m, width, hidden, act):
    """Against the hidden values of exact sums, held in float64's own way.  A value that is off by d of itself lands on the other side of a border of the grid with a probability of d over the
    step, and is then off by a step.  Float32 sums of `width` products of either sign are off by about 2^-24 sqrt(width) <= 2^-19 of themselves, the activation by 2^-20: with a step of 2^-3.5, the
    middle, about 2^-15 of the values cross, which is 2^-7.5 of a step, 2^-11, in 2-norm.  The result is rounded by up to 2^-11, evenly spread.  Both together, doubled: 2 * 2^-11 sqrt(1 + 1/3)."""
    g = torch.Generator(device="cuda").manual_seed(m + hidden)
    rand = lambda *s: torch.randn(s, generator=g, device="cuda")  # noqa: E731
    rows, w_in = sjd.op_norm_f8(rand(m, width), norm="rms"), sjd.op_norm_f8(rand(2 * hidden, width) * width ** -0.5, norm="none")
    w_out = sjd.op_norm_f8(rand(130, hidden) * hidden ** -0.5, norm="none")
    got = sjd.op_gated_mlp_f8(rows, w_in, w_out, activation=act, dtype=F16)
    at = torch.arange(0, m, max(1, m // 300))
    val = lambda r, pick=None: ref.values(r.codes[slice(None) if pick is None else pick].cpu(), r.scales[slice(None) if pick is None else pick].cpu(), r.width)  # noqa: E731
    z = val(rows, at.cuda()) @ val(w_in).T
    h = ref.values(*ref.hold((ref.activation(z[:, :hidden], act) * z[:, hidden:]).float()), hidden)
    want = h @ val(w_out).T
    assert float((got[at.cuda()].cpu().double() - want).norm() / want.norm()) <= 2 * 2.0 ** -11 * math.sqrt(4 / 3)


# 32x32 tiles (one and two a CU), 64x64 in two parts of k, 128x64, 64x64 and 128x64 several to a CU, 128x128 one and two to a CU
@pytest.mark.parametrize("m,n", [(200, 300), (500, 900), (900, 1027), (1500, 1027), (700, 2901), (1300, 2051), (3000, 1203), (1300, 4099), (4001, 2003), (9001, 1027)])
@pytest.mark.parametrize("k", [128, 700])
def test_projection_into_the_stream_by_every_tile(m, n, k):
    """Odd numbers of outputs, so that the last columns are a part of the last eight, in rows that begin anywhere in wider ones."""
    xc, xs, x = _integers_gpu(m, m, k, top=2)
    wc, ws, w = _integers_gpu(n, n, k, top=2)
    bias = (torch.arange(n, device="cuda") % 13 - 6).float()
    wide = (torch.arange(m * (n + 3), device="cuda") % 101 - 50).float().view(m, n + 3)
    want = wide.double()
    want[:, 1:1 + n] += x @ w.T + bias.double()
    got = sjd.op_linear_f8(sjd.F8Rows(xc, xs, k), sjd.F8Rows(wc, ws, k), bias=bias, resid=wide[:, 1:1 + n])
    assert got.data_ptr() == wide[:, 1:].data_ptr() and torch.equal(wide.double(), want)


@pytest.mark.parametrize("m,width,hidden", LAUNCHES)
@pytest.mark.parametrize("act", ["silu", "gelu"])
def test_gated_block_into_the_stream_and_into_rows_of_a_larger_tensor(m, width, hidden, act):
    """A gate that is 128 or nothing, `up` of small integers: hidden values are held as they are, and the weight behind them is of integers too."""
    g = _gen(m + hidden)
    n = 133
    x = torch.zeros(m, width)
    x[:, 0] = 1
    x[:, 1:4] = torch.randint(-2, 3, (m, 3), generator=g)
    gate = torch.zeros(hidden, width)
    gate[:, 0] = torch.where(torch.rand(hidden, generator=g) < 0.3, -192.0, 128.0)
    up = torch.zeros(hidden, width)
    up[:, 1:4] = torch.randint(0, 2, (hidden, 3), generator=g)
    w_out = torch.randint(-2, 3, (n, hidden), generator=g).float()
    h = torch.clamp(x @ gate.T, min=0) * (x @ up.T)
    assert torch.equal(ref.values(*ref.hold(h[:50]), hidden), h[:50].double())
    want = (h.cuda().double() @ w_out.cuda().double().T)
    rows, w_in, w_o = _rows(*ref.hold(x), width), _rows(*ref.hold(torch.cat((gate, up))), width), _rows(*ref.hold(w_out), hidden)
    wide = (torch.arange(m * (n + 6), device="cuda") % 64 * 128.0).view(m, n + 6)
    after = wide.double()
    after[:, 2:2 + n] += want
    got = sjd.op_gated_mlp_f8(rows, w_in, w_o, activation=act, resid=wide[:, 2:2 + n])
    assert got.data_ptr() == wide[:, 2:].data_ptr() and torch.equal(wide.double(), after)
    for dtype in TYPES:
        out = torch.full((m + 2, n + 6), 3.0, dtype=dtype, device="cuda")
        assert sjd.op_gated_mlp_f8(rows, w_in, w_o, activation=act, out=out[1:-1, 2:2 + n]).dtype is dtype
        assert torch.equal(out[1:-1, 2:2 + n], want.to(F32).to(dtype))
        out[1:-1, 2:2 + n] = 3
        assert (out == 3).all()

"""The 8-bit operators where a call is unlike the others: offsets beyond 32 bits, rows of NaN beside others, streams, captured graphs, a layer's calls together."""
import math

import pytest
import torch

import f8_reference as ref
import paper_2505_24791_amd as sjd
from test_gpu_f8 import BF16, F16, F32, TYPES, _gate_integers, _gen, _integers, _integers_gpu, _randn, _rows

pytestmark = pytest.mark.gpu


def _room(gigabytes):
    free = torch.cuda.mem_get_info()[0]
    if free < gigabytes * 1e9:
        pytest.skip(f"needs {gigabytes} GB of device memory")


# ------------------------------------------------------------------------------------------------ beyond 32 bits

def test_norm_of_rows_beyond_4_gb():
    _room(12)
    g = torch.Generator(device="cuda").manual_seed(1)
    x = torch.empty((140000, 8200), dtype=F32, device="cuda")              # 4.6 GB; its 8 bits 1.2 GB
    x[:] = torch.arange(140000, device="cuda").unsqueeze(1) % 7
    x[-3:] = torch.randn((3, 8200), generator=g, device="cuda")
    got = sjd.op_norm_f8(x, norm="rms")
    tail = sjd.op_norm_f8(x[-3:], norm="rms")
    assert torch.equal(got.codes[-3:], tail.codes) and torch.equal(got.scales[-3:], tail.scales)
    assert torch.equal(got.codes[8], got.codes[1]) and not torch.equal(got.codes[8], got.codes[7])
    out = torch.empty((140000, 8200), dtype=F32, device="cuda")
    sjd.op_f8_read(got, F32, out=out)
    assert torch.equal(out[-3:], sjd.op_f8_read(tail, F32))


@pytest.mark.parametrize("k", [128, 256])
@pytest.mark.parametrize("dtype", TYPES)
def test_results_beyond_4_gb(k, dtype):
    """530000 x 4160: by 128x128 tiles (one k-tile, float32) and by the kernel that walks over tiles."""
    m, n = 530000, 4160
    _room(14)
    xc, xs, x = _integers_gpu(3, 1000, k)
    wc, ws, w = _integers_gpu(4, n, k)
    at = torch.randint(0, 1000, (m,), generator=torch.Generator(device="cuda").manual_seed(5), device="cuda")
    got = sjd.op_linear_f8(sjd.F8Rows(xc[at], xs[at], k), sjd.F8Rows(wc, ws, k), dtype=dtype)
    want = (x @ w.T).to(F32).to(dtype)
    for r in (0, 262143, 516221, 516222, m - 1):
        assert torch.equal(got[r], want[at[r]]), r
    for a in range(0, m, 53000):
        assert torch.equal(got[a:a + 53000], want[at[a:a + 53000]]), a


@pytest.mark.parametrize("dtype", TYPES)
def test_operands_beyond_4_gb(dtype):
    """A weight of 600000 outputs by 8192, then as the rows."""
    n, k = 600000, 8192
    _room(16)
    wc = torch.zeros((n, k), dtype=torch.uint8, device="cuda")
    ws = torch.full((n, 64), 127, dtype=torch.uint8, device="cuda")
    places = torch.arange(n, device="cuda") * 7919 % k
    wc[torch.arange(n, device="cuda"), places] = 0x38 + (torch.arange(n, device="cuda") % 2 * 8).to(torch.uint8)        # one 1 or 2 a row
    xc, xs, x = _integers(_gen(1), 20, k)
    rows, weight = _rows(xc, xs, k), sjd.F8Rows(wc, ws, k)
    want = (x.cuda()[:, places] * (1 + torch.arange(n, device="cuda") % 2)).to(F32).to(dtype)
    assert torch.equal(sjd.op_linear_f8(rows, weight, dtype=dtype), want)
    assert torch.equal(sjd.op_linear_f8(weight, rows, dtype=dtype), want.T)


# ------------------------------------------------------------------------------------------------ rows beside others

@pytest.mark.parametrize("m,n", [(40, 70), (300, 700), (1000, 1000), (3000, 1200), (9000, 2304), (9000, 2303)])
@pytest.mark.parametrize("dtype", TYPES)
def test_a_row_of_nan_is_one_row(m, n, dtype):
    k = 384
    xc, xs, x = _integers_gpu(m, m, k)
    wc, ws, w = _integers_gpu(n, n, k)
    xc[m - 2, 5] = 0x7f
    wc[n - 3, 300] = 0xff
    got = sjd.op_linear_f8(sjd.F8Rows(xc, xs, k), sjd.F8Rows(wc, ws, k), dtype=dtype)
    want = (x @ w.T).to(F32).to(dtype)
    bad = torch.zeros_like(want, dtype=torch.bool)
    bad[m - 2] = True
    bad[:, n - 3] = True
    assert torch.equal(torch.isnan(got), bad)
    assert torch.equal(got[~bad], want[~bad])


@pytest.mark.parametrize("m,hidden", [(5, 200), (300, 640), (9000, 2304)])
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("act", ["silu", "gelu"])
def test_hidden_values_beyond_float32_poison_their_row_alone(m, hidden, dtype, act):
    width = 256
    g = _gen(hidden)
    (xc, xs), (wc, ws) = _gate_integers(g, 50, width, hidden)
    at = torch.arange(m) % 49
    at[m // 2] = 49
    xs = xs.clone()
    xs[49, :2] += 70                                                       # gate and up sums of one row times 2^70
    z = ref.values(xc, xs, width) @ ref.values(wc, ws, width).T
    h = torch.clamp(z[:, :hidden], min=0) * z[:, hidden:]
    assert (h[49].abs() > torch.finfo(F32).max).any()
    held = ref.values(*ref.hold(h[:49]), hidden)
    pick = torch.randint(0, hidden, (64,), generator=g)
    w_out = torch.zeros(64, hidden)
    w_out[torch.arange(64), pick] = 1
    got = sjd.op_gated_mlp_f8(_rows(xc[at], xs[at], width), _rows(wc, ws, width), _rows(*ref.hold(w_out), hidden), activation=act, dtype=dtype).cpu()
    assert torch.isnan(got[m // 2]).all()
    others = torch.arange(m) != m // 2
    assert torch.equal(got[others], held[:, pick].to(F32).to(dtype)[at[others]])


def test_no_rows_and_one_value():
    w = _rows(*ref.hold(torch.ones(5, 200)), 200)
    none = sjd.op_norm_f8(torch.empty((0, 200), device="cuda"))
    assert sjd.op_linear_f8(none, w).shape == (0, 5) and sjd.op_f8_read(none, BF16).shape == (0, 200) and none.codes.shape == (0, 256) and none.scales.shape == (0, 4)
    w_in, w_out = _rows(*ref.hold(torch.ones(6, 200)), 200), _rows(*ref.hold(torch.ones(7, 3)), 3)
    assert sjd.op_gated_mlp_f8(none, w_in, w_out).shape == (0, 7)
    x = _rows(*ref.hold(torch.ones(4, 200)), 200)
    assert sjd.op_linear_f8(x, _rows(torch.empty((0, 256), dtype=torch.uint8), torch.empty((0, 4), dtype=torch.uint8), 200)).shape == (4, 0)
    one = sjd.op_norm_f8(torch.full((1, 1), -3.0, device="cuda"), norm="rms")
    assert float(sjd.op_linear_f8(one, one, dtype=F32)) == 1.0


def test_the_residual_may_be_the_rows_themselves():
    x = _randn(_gen(3), 33, 777)
    d = x.cuda()
    got = sjd.op_norm_f8(d, resid=d, norm="layer")
    y, after = ref.normed(x, x, "layer", None, None, 1e-6)
    assert torch.equal(d.cpu(), after) and torch.equal(got.codes.cpu(), ref.hold(y)[0])


# ------------------------------------------------------------------------------------------------ streams and graphs

def _layer(seed, n, dim=512, heads=8, hidden=700):
    """A layer's tensors for n rows that are the last tokens of n sequences."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    rand = lambda *s: torch.randn(s, generator=g, device="cuda")  # noqa: E731
    held = lambda outs, width: sjd.op_norm_f8(rand(outs, width) * width ** -0.5, norm="none")  # noqa: E731
    d = dim // heads
    cache = sjd.Kv4Cache.zeros(n, heads, d, BF16)
    old = torch.arange(n, device="cuda", dtype=torch.int32) * 64
    for t in range(5):                                                     # five tokens that are there already
        sjd.op_kv4_write(cache, rand(n, heads, d).bfloat16(), rand(n, heads, d).bfloat16(), old + t)
    return {"x": rand(n, dim).bfloat16(), "stream": rand(n, dim), "gains": [1 + 0.1 * rand(dim) for _ in range(2)], "qkv": held(3 * dim, dim), "bias": rand(3 * dim), "o": held(dim, dim),
            "w_in": held(2 * hidden, dim), "w_out": held(dim, hidden), "cache": cache, "slot": old + 5, "table": torch.arange(n, device="cuda", dtype=torch.int32).unsqueeze(1),
            "len": torch.full((n,), 6, dtype=torch.int32, device="cuda"), "heads": heads, "d": d,
            "opts": sjd.QkOpts(norm="rms", rot_dim=d, axis_pairs=(d // 2,), freq=torch.logspace(0, -3, d // 2).cuda()), "pos": torch.full((n, 1), 5, dtype=torch.int32, device="cuda")}


def _run_layer(p):
    """One layer for single tokens, in 8 bits: what it gives and what lies in between."""
    n, heads, d, s = p["x"].shape[0], p["heads"], p["d"], p["stream"]
    a = sjd.op_norm_f8(p["x"], resid=s, gain=p["gains"][0])
    qkv = sjd.op_linear_f8(a, p["qkv"], bias=p["bias"], dtype=BF16).view(n, 3 * heads, d)
    q = sjd.op_kv4_write(p["cache"], qkv[:, heads:2 * heads], qkv[:, 2 * heads:], p["slot"], opts=p["opts"], pos=p["pos"], q=qkv[:, :heads])
    o = sjd.op_kv4_attention(p["cache"], q, p["table"], p["len"], max_kv=6)
    b = sjd.op_norm_f8(o.view(n, heads * d), norm="none")
    y = sjd.op_linear_f8(b, p["o"], dtype=BF16)
    c = sjd.op_norm_f8(y, resid=s, gain=p["gains"][1])
    z = sjd.op_gated_mlp_f8(c, p["w_in"], p["w_out"], dtype=BF16)
    return {"a": a, "qkv": qkv, "o": o, "b": b, "y": y, "c": c, "z": z, "stream": s}


@pytest.mark.parametrize("n", [3, 70, 600])
def test_a_layer_together(n):
    """Each call against its float64 form on what it was given on the device."""
    p = _layer(n, n)
    x, s0 = p["x"].cpu(), p["stream"].cpu().clone()
    r = _run_layer(p)
    val = lambda rows: ref.values(rows.codes.cpu(), rows.scales.cpu(), rows.width)  # noqa: E731
    y, s1 = ref.normed(x, s0, "rms", p["gains"][0].cpu(), None, 1e-6)
    assert torch.equal(r["a"].codes.cpu(), ref.hold(y)[0])

    def near(got, a, w, bias=None):
        want, mag = a @ w.T, a.abs() @ w.abs().T
        if bias is not None:
            want, mag = want + bias.double(), mag + bias.double().abs()
        far = (a.shape[1] + 2) * 2.0 ** -24 * mag + ref.dropped(a, w)
        far = far + torch.finfo(BF16).eps / 2 * (want.abs() + far)
        assert ((got.cpu().double() - want).abs() <= far).all()
    near(r["qkv"].reshape(n, -1), val(r["a"]), val(p["qkv"]), p["bias"].cpu())
    assert torch.equal(r["b"].codes.cpu(), ref.hold(r["o"].view(n, -1).cpu())[0])
    near(r["y"], val(r["b"]), val(p["o"]))
    y, s2 = ref.normed(r["y"].cpu(), s1, "rms", p["gains"][1].cpu(), None, 1e-6)
    assert torch.equal(r["c"].codes.cpu(), ref.hold(y)[0]) and torch.equal(r["stream"].cpu(), s2)
    h = val(r["c"]) @ val(p["w_in"]).T
    want = (ref.activation(h[:, :700], "silu") * h[:, 700:]) @ val(p["w_out"]).T
    assert float((r["z"].cpu().double() - want).norm() / want.norm()) <= 2 * 2.0 ** -4 / math.sqrt(3)     # hidden values to four bits, evenly spread


@pytest.mark.parametrize("n", [3, 600])
def test_a_captured_layer_replayed_between_eager_calls(n):
    p = _layer(7, n)
    stream0 = p["stream"].clone()
    side = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        _run_layer(p)                                                      # what a first call loads is loaded before
        side.synchronize()
        with torch.cuda.graph(graph, stream=side):
            p["stream"].copy_(stream0)
            r = _run_layer(p)
    torch.cuda.current_stream().wait_stream(side)
    g = torch.Generator(device="cuda").manual_seed(9)
    for i in range(4):
        p["x"].copy_(torch.randn(p["x"].shape, generator=g, device="cuda"))
        graph.replay()
        got = {k: (v.codes if isinstance(v, sjd.F8Rows) else v).clone() for k, v in r.items()}
        p["stream"].copy_(stream0)
        want = _run_layer(p)
        torch.cuda.synchronize()
        for k, v in want.items():
            assert torch.equal(got[k], v.codes if isinstance(v, sjd.F8Rows) else v), (i, k)


@pytest.mark.parametrize("m", [3, 65, 600, 9000])
def test_two_captured_graphs_replayed_at_once(m):
    """Gated blocks on two streams: each has its own hidden rows."""
    g = torch.Generator(device="cuda").manual_seed(m)
    graphs, outs, wants, streams = [], [], [], [torch.cuda.Stream() for _ in range(2)]
    for s in streams:
        x = sjd.op_norm_f8(torch.randn((m, 384), generator=g, device="cuda"), norm="rms")
        w_in = sjd.op_norm_f8(torch.randn((2 * 2304, 384), generator=g, device="cuda") * 0.05, norm="none")
        w_out = sjd.op_norm_f8(torch.randn((200, 2304), generator=g, device="cuda") * 0.02, norm="none")
        call = lambda x=x, w_in=w_in, w_out=w_out: sjd.op_gated_mlp_f8(x, w_in, w_out, dtype=BF16)  # noqa: E731
        wants.append(call().clone())
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.graph(graph, stream=s):
            for _ in range(3):
                out = call()
        graphs.append((graph, x, w_in, w_out))
        outs.append(out)
    for _ in range(3):
        for (graph, *_), s in zip(graphs, streams):
            with torch.cuda.stream(s):
                graph.replay()
        torch.cuda.synchronize()
        for out, want in zip(outs, wants):
            assert torch.equal(out, want)
            out.zero_()


@pytest.mark.parametrize("m", [5, 300, 9000])
def test_calls_on_a_stream_of_their_own(m):
    """The rows are made on the stream that the call is on, behind work that takes long."""
    side = torch.cuda.Stream()
    g = torch.Generator(device="cuda").manual_seed(m)
    x = torch.randn((m, 640), generator=g, device="cuda")
    w = sjd.op_norm_f8(torch.randn((2304, 640), generator=g, device="cuda") * 0.04, norm="none")
    want = sjd.op_linear_f8(sjd.op_norm_f8(2 * x, norm="rms"), w)
    big = torch.randn((4096, 4096), device="cuda")
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        late = big
        for _ in range(4):
            late = late @ big * 1e-2
        y = x * (2 + 0 * late[0, 0].nan_to_num(0, 0, 0))
        got = sjd.op_linear_f8(sjd.op_norm_f8(y, norm="rms"), w)
    side.synchronize()
    assert torch.equal(got, want)


def test_the_same_call_gives_the_same_bits():
    g = torch.Generator(device="cuda").manual_seed(2)
    for m, n, k in ((7, 100, 1000), (100, 2304, 768), (700, 1100, 2050), (9000, 2304, 768)):
        x = sjd.op_norm_f8(torch.randn((m, k), generator=g, device="cuda"), norm="rms")
        w = sjd.op_norm_f8(torch.randn((n, k), generator=g, device="cuda"), norm="none")
        for dtype in TYPES:
            first = sjd.op_linear_f8(x, w, dtype=dtype)
            assert all(torch.equal(sjd.op_linear_f8(x, w, dtype=dtype), first) for _ in range(5)), (m, n, k, dtype)


def test_a_weight_whose_storage_is_replaced():
    a, b = _integers_gpu(1, 50, 300), _integers_gpu(2, 50, 300)
    x = _integers_gpu(3, 9, 300)
    rows, weight = sjd.F8Rows(x[0], x[1], 300), sjd.F8Rows(a[0], a[1], 300)
    assert torch.equal(sjd.op_linear_f8(rows, weight, dtype=F32).double(), x[2] @ a[2].T)
    weight.codes.data, weight.scales.data = b[0], b[1]
    assert torch.equal(sjd.op_linear_f8(rows, weight, dtype=F32).double(), x[2] @ b[2].T)


def test_as_many_rows_as_are_read_back_at_once():
    """2^25 - 1 rows of 640, the most of that width: the first, the last and some between differ from the others."""
    n, width = (1 << 25) - 1, 640
    _room(72)
    codes = torch.full((n, width), 0x38, dtype=torch.uint8, device="cuda")
    scales = torch.full((n, 8), 127, dtype=torch.uint8, device="cuda")
    marks = [0, 1, n // 2, n // 2 + 1, n - 3, n - 2, n - 1]
    for i, r in enumerate(marks):
        codes[r, i::3] = 0x40 + 8 * i                                      # 2, 4, 8 ..
        scales[r, i % 5] = 120
    out = torch.empty((n, width), dtype=F16, device="cuda")
    sjd.op_f8_read(sjd.F8Rows(codes, scales, width), F16, out=out)
    want = ref.values(codes[marks].cpu(), scales[marks].cpu(), width).half()
    assert torch.equal(out[marks].cpu(), want)
    out[marks] = 1
    for a in range(0, n, 1 << 22):
        assert bool((out[a:a + (1 << 22)] == 1).all()), a


@pytest.mark.parametrize("m,n,k", [(4, 40, 128), (40, 300, 256), (900, 1027, 256), (3000, 1203, 256), (9000, 2304, 256)])
@pytest.mark.parametrize("dtype", TYPES)
def test_scales_at_the_ends_of_their_range(m, n, k, dtype):
    """One product a result, of scales 2^e and 2^-e: exact down to the smallest code with e = -120, and up to what float32 has; beyond that infinite where products are exact (float32)."""
    codes = torch.tensor([0x01, 0x02, 0x03, 0x05, 0x07, 0x08, 0x0f, 0x38, 0x70, 0x77, 0x78, 0x7d, 0x7e, 0x81, 0xfe], dtype=torch.uint8)
    for e in (-120, -119, -118, 118, 119, 120):
        xc, wc = torch.zeros((m, k), dtype=torch.uint8), torch.zeros((n, k), dtype=torch.uint8)
        xc[:, 3], wc[:, 3] = codes[torch.arange(m) % len(codes)], codes[torch.arange(n) // 3 % len(codes)]
        xs, ws = torch.full((m, 4), 127 + e, dtype=torch.uint8), torch.full((n, 4), 127 - e, dtype=torch.uint8)
        x, w = ref.values(xc, xs, k), ref.values(wc, ws, k)
        want = x[:, 3:4] * w[:, 3]
        if dtype is F32:
            x, w = (torch.where(v.abs() >= 2.0 ** 128, math.inf * v.sign(), v) for v in (x[:, 3:4], w[:, 3]))
            far = torch.isinf(x) | torch.isinf(w)
            want = torch.where(far, math.nan, want)                        # beside zeros in the other channels: infinite or not a number
        want = want.to(F32).to(dtype)
        got = sjd.op_linear_f8(_rows(xc, xs, k), _rows(wc, ws, k), dtype=dtype).cpu()
        fine = ~torch.isnan(want)
        assert torch.equal(got[fine], want[fine]), e
        assert not torch.isfinite(got[~fine]).any(), e
        assert m < len(codes) or bool((~fine).any()) == (dtype is F32 and abs(e) == 120), e        # all codes are there


@pytest.mark.parametrize("m,n", [(1, 128257), (64, 65536), (300, 40000), (700, 33000)])
@pytest.mark.parametrize("dtype", [BF16, F16])
def test_few_rows_by_many_outputs(m, n, dtype):
    """One to three panels of 256 rows, which the kernel that walks over tiles would leave to as many XCDs; the gate too."""
    k = 256
    xc, xs, x = _integers_gpu(m, m, k)
    wc, ws, w = _integers_gpu(n, n, k)
    bias = (torch.arange(n, device="cuda") % 13 - 6).float()
    got = sjd.op_linear_f8(sjd.F8Rows(xc, xs, k), sjd.F8Rows(wc, ws, k), bias=bias, dtype=dtype)
    assert torch.equal(got, (x @ w.T + bias.double()).to(F32).to(dtype))
    hidden = min(n // 2, 16400)
    g = _gen(n)
    (gc, gs), (ic, is_) = _gate_integers(g, min(m, 60), k, hidden)
    at = torch.arange(m) % min(m, 60)
    z = ref.values(gc, gs, k) @ ref.values(ic, is_, k).T
    held = ref.values(*ref.hold(torch.clamp(z[:, :hidden], min=0) * z[:, hidden:]), hidden)
    pick = torch.randint(0, hidden, (90,), generator=g)
    w_out = torch.zeros(90, hidden)
    w_out[torch.arange(90), pick] = 1
    got = sjd.op_gated_mlp_f8(_rows(gc[at], gs[at], k), _rows(ic, is_, k), _rows(*ref.hold(w_out), hidden), dtype=dtype).cpu()
    assert torch.equal(got, held[:, pick].to(F32).to(dtype)[at])

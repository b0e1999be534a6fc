"""Head norms with rotation, the 4-bit key/value cache and attention over it, through the binding, against plain float64 forms.
Needs an MI355X.

Bounds.  ``half`` is half a step of the rows' type relative to a value (2^-11, 2^-8, 2^-24).  Norms and rotation are computed in
float64 and rounded to float32 and then to the type: half (1 + 2^-12) of the value.  What the cache holds is exact.  Attention rounds
its probabilities to the type (half each, of numerator and denominator alike: half (sum p |v| / sum p + |o|)), the result once more, and
sums in float32: scores over dim channels, sums over the keys, 2^-24 of the magnitudes for each term."""
import numpy as np
import pytest

from kv4_reference import attention, held, norm_rotate

pytestmark = [pytest.mark.gpu, pytest.mark.timeout(300)]

HALF = {"float16": 2.0 ** -11, "bfloat16": 2.0 ** -8, "float32": 2.0 ** -24}
TINY = {"float16": 2.0 ** -25, "bfloat16": 0.0, "float32": 0.0}          # half a step of the subnormals
TYPES = list(HALF)


@pytest.fixture(scope="module")
def torch_cuda():
    import torch
    assert torch.cuda.is_available(), "these tests need the GPU"
    return torch


def _rows(torch, rng, n, h, d, name, spread=1.0, pad=0, offset=0):
    """Rows [n, h, d] of a wider allocation: pad elements between them, the first one offset elements in."""
    base = torch.zeros(n * (h * d + pad) + offset + 8, dtype=getattr(torch, name), device="cuda")
    t = base[offset:offset + n * (h * d + pad)].view(n, h * d + pad)[:, :h * d].unflatten(1, (h, d))
    t.copy_(torch.from_numpy(rng.standard_normal((n, h, d)) * spread))
    return t


def _f64(t):
    return t.detach().double().cpu().numpy()


def _opts(torch, sjd, rng, dim, norm, rot, adjacent, sections, gains=True):
    g = {}
    if norm != "none" and gains:
        g = {k: (rng.standard_normal(dim) * 0.2 + 1).astype(np.float32) for k in ("q_gain", "k_gain")}
    if norm == "layer":
        g.update({k: (rng.standard_normal(dim) * 0.2).astype(np.float32) for k in ("q_shift", "k_shift")})
    freq = np.concatenate([10000.0 ** (-np.arange(p) / max(p, 1)) for p in sections]).astype(np.float32) if rot else None
    o = sjd.QkOpts(norm=norm, eps=1e-5, rot_dim=rot, adjacent=adjacent, axis_pairs=sections,
                   freq=None if freq is None else torch.from_numpy(freq).cuda(), **{k: torch.from_numpy(v).cuda() for k, v in g.items()})
    ref = lambda side: dict(norm=norm, eps=1e-5, gain=g.get(side + "_gain"), shift=g.get(side + "_shift"), rot=rot, adjacent=adjacent,
                            axis_pairs=sections, freq=freq)
    return o, ref


def _near(got, want, name, what):
    got = _f64(got)
    bound = HALF[name] * (1 + 2.0 ** -12) * np.abs(want) + TINY[name] + 1e-13 * np.abs(want).max(-1, keepdims=True)
    worst = np.max(np.abs(got - want) / np.maximum(bound, 1e-300))
    assert worst <= 1.0, (what, worst)


ROPE = [
    # rows, heads, kv heads, dim, norm, rot, adjacent, pairs of the axes, padding between rows, offset of the first
    (1, 4, 4, 64, "rms", 64, False, (32,), 0, 0),
    (33, 12, 12, 64, "rms", 64, False, (16, 16), 64, 0),
    (7, 6, 2, 128, "layer", 128, True, (16, 24, 24), 1, 1),
    (4100, 3, 1, 32, "rms", 16, False, (8,), 3, 5),
    (5, 8, 1, 256, "layer", 256, False, (40, 40, 40, 8), 0, 2),
    (130, 2, 2, 80, "rms", 40, True, (7, 13), 0, 0),
    (9, 1, 1, 8, "none", 8, False, (1, 3), 0, 0),
    (17, 5, 5, 48, "rms", 0, False, (), 7, 3),
    (64, 16, 4, 64, "none", 32, True, (0, 16), 0, 0),
]


@pytest.mark.parametrize("name", TYPES)
@pytest.mark.parametrize("case", ROPE, ids=lambda c: "x".join(map(str, c[:4])) + c[4])
def test_norm_and_rotation(torch_cuda, name, case):
    import paper_2505_24791_amd as sjd
    torch = torch_cuda
    n, H, KV, dim, norm, rot, adjacent, sections, pad, offset = case
    rng = np.random.default_rng(n * 100 + dim)
    q, k = (_rows(torch, rng, n, h, dim, name, 1.5, pad, offset) for h in (H, KV))
    o, ref = _opts(torch, sjd, rng, dim, norm, rot, adjacent, sections)
    pos = rng.integers(-50, 3000, (n, max(1, len(sections)))).astype(np.int32)
    dpos = torch.from_numpy(pos).cuda() if rot else None
    wq, wk = norm_rotate(_f64(q), pos, **ref("q")), norm_rotate(_f64(k), pos, **ref("k"))
    gq, gk = sjd.op_qk_norm_rope(q, k, dpos, o)
    _near(gq, wq, name, "q")
    _near(gk, wk, name, "k")
    # one side alone, and in place
    only, none = sjd.op_qk_norm_rope(None, k, dpos, o)[::-1]
    assert none is None and torch.equal(only, gk)
    sjd.op_qk_norm_rope(q, k, dpos, o, q_out=q, k_out=k)
    assert torch.equal(q, gq) and torch.equal(k, gk)


def test_angles_of_far_positions(torch_cuda):
    """Positions to the ends of int32, frequencies up to several radians a step."""
    import paper_2505_24791_amd as sjd
    torch = torch_cuda
    rng = np.random.default_rng(3)
    pos = np.array([[0], [1], [-1], [2 ** 31 - 1], [-2 ** 31], [123456789], [16777217], [99999999]], np.int32)
    q = _rows(torch, rng, len(pos), 2, 64, "float32")
    freq = np.concatenate([[3.0, 1.0, 0.7, 1e-3], rng.uniform(1e-6, 2, 28)]).astype(np.float32)
    o = sjd.QkOpts(norm="none", rot_dim=64, axis_pairs=(32,), freq=torch.from_numpy(freq).cuda())
    got, _ = sjd.op_qk_norm_rope(q, None, torch.from_numpy(pos).cuda(), o)
    want = norm_rotate(_f64(q), pos, norm="none", eps=0, gain=None, shift=None, rot=64, adjacent=False, axis_pairs=(32,), freq=freq)
    # the reference's own angle is good to 2^-64 of 2^31 turns of three radians
    assert np.abs(_f64(got) - want).max() <= (HALF["float32"] + 1e-9) * np.abs(_f64(q)).max() * 2


def test_rows_of_zeros_and_of_no_norm(torch_cuda):
    import paper_2505_24791_amd as sjd
    torch = torch_cuda
    q = torch.zeros((3, 2, 64), device="cuda")
    for norm in ("rms", "layer"):
        got, _ = sjd.op_qk_norm_rope(q, None, None, sjd.QkOpts(norm=norm, eps=1e-6))
        assert torch.equal(got, q)
    got, none = sjd.op_qk_norm_rope(q[:0], None, None, sjd.QkOpts())
    assert got.shape == (0, 2, 64) and none is None


# ---- the cache ----

def _special(rng, n, h, dim, name):
    """Rows with what a group can hold: ties of the grid, zeros, one value alone, the type's smallest and largest."""
    x = rng.standard_normal((n, h, dim))
    flat = x.reshape(-1, 32)
    grid = np.array([0, .25, .5, .75, 1, 1.25, 1.5, 1.75, 2, 2.5, 3, 3.5, 4, 5, 6, 6.5, 7])
    top, low = {"float16": (65504.0, 2.0 ** -24), "bfloat16": (3.3895e38, 1e-40), "float32": (3.4028234e38, 1e-45)}[name]
    for i in range(len(flat)):
        m = i % 9
        if m == 0:
            flat[i] = rng.choice(grid, 32) * rng.choice([-1, 1], 32) * 2.0 ** rng.integers(-9, 9)
        elif m == 1:
            flat[i] = 0.0
        elif m == 2:
            flat[i] = 0.0
            flat[i, i % 32] = -1.75 * 2.0 ** rng.integers(-5, 5)
        elif m == 3:
            flat[i] *= top / 8
        elif m == 4:
            flat[i] = rng.choice([top, -top, top / 2, 0.0, 1.0], 32)
        elif m == 5:
            flat[i] = low * rng.integers(-9, 9, 32)
        elif m == 6:
            flat[i] = np.where(rng.random(32) < 0.5, -0.0, 1e-3)
        elif m == 7:
            flat[i] *= 2.0 ** rng.integers(-14, 14)
    return x


@pytest.mark.parametrize("name", TYPES)
@pytest.mark.parametrize("dim,kv,n", [(32, 3, 70), (64, 1, 1), (64, 4, 200), (128, 2, 129), (256, 2, 65)])
def test_written_tokens_read_back_as_the_format_says(torch_cuda, name, dim, kv, n):
    import paper_2505_24791_amd as sjd
    torch = torch_cuda
    rng = np.random.default_rng(dim + n)
    k, v = (torch.from_numpy(_special(rng, n, kv, dim, name)).to(getattr(torch, name)).cuda() for _ in range(2))
    pages = n // 64 + 3
    cache = sjd.Kv4Cache(torch.full((pages, kv, 68 * dim), 0xA7, dtype=torch.uint8, device="cuda"), k.dtype)
    before = sjd.op_kv4_read(cache, torch.arange(pages * 64, dtype=torch.int32, device="cuda"))
    slot = torch.from_numpy(rng.permutation(pages * 64)[:n].astype(np.int32)).cuda()
    out = slot.clone()
    slot[::7] = -1
    if n > 20:
        slot[3], slot[10], slot[11] = pages * 64, 2 ** 31 - 1, -2 ** 31
    sjd.op_kv4_write(cache, k, v, slot)
    gk, gv = sjd.op_kv4_read(cache, out)
    in_it = ((slot >= 0) & (slot < pages * 64)).cpu().numpy()
    for got, x, old in ((gk, k, before[0]), (gv, v, before[1])):
        want = held(_f64(x), name)
        assert np.array_equal(_f64(got)[in_it], want[in_it])
        assert torch.equal(got[~in_it].view(torch.uint8), old[out.long()][~in_it].view(torch.uint8))     # left as it was
    # every other token too
    rest = torch.ones(pages * 64, dtype=torch.bool, device="cuda")
    rest[out.long()] = False
    after = sjd.op_kv4_read(cache, torch.arange(pages * 64, dtype=torch.int32, device="cuda"))
    for a, b in zip(after, before):
        assert torch.equal(a[rest].view(torch.uint8), b[rest].view(torch.uint8))
    # a slot outside the cache reads as zeros
    z = sjd.op_kv4_read(cache, torch.tensor([-1, pages * 64, 2 ** 31 - 1, -2 ** 31], dtype=torch.int32, device="cuda"))
    assert not z[0].any() and not z[1].any()


@pytest.mark.parametrize("dim", [32, 64, 128, 256])
@pytest.mark.parametrize("order", ["on", "shifted", "holes", "swapped", "backward", "ends"])
def test_tokens_in_and_out_of_order(torch_cuda, dim, order):
    """Runs of tokens from page starts and from elsewhere, with rows left out in between, pairs swapped, backward, and slots around the ends of the cache."""
    import paper_2505_24791_amd as sjd
    torch = torch_cuda
    rng = np.random.default_rng(dim)
    n, kv = 193, 2
    k, v = (torch.from_numpy(_special(rng, n, kv, dim, "bfloat16")).to(torch.bfloat16).cuda() for _ in range(2))
    t = np.arange(n)
    slots = {"on": t, "shifted": t + 3, "holes": np.where(t % 5 == 2, -1, t), "swapped": t ^ 1, "backward": n + 2 - t, "ends": t - 2}[order].astype(np.int64)
    pages = 4
    if order == "ends":
        slots = np.where(t >= 100, slots + pages * 64 - 150, slots)               # 98 .. before the end and past it
        slots[[7, 8, 9, 10, 11, 12]] = [-2 ** 31, 2 ** 31 - 1, -2 ** 31, -2 ** 31 + 1, -2 ** 31 + 2, -2 ** 31 + 3]
    cache = sjd.Kv4Cache(torch.full((pages, kv, 68 * dim), 0x5A, dtype=torch.uint8, device="cuda"), torch.bfloat16)
    everything = torch.arange(pages * 64, dtype=torch.int32, device="cuda")
    before = [_f64(x) for x in sjd.op_kv4_read(cache, everything)]
    slot = torch.from_numpy(slots.astype(np.int32)).cuda()
    sjd.op_kv4_write(cache, k, v, slot)
    fused = sjd.Kv4Cache(torch.full_like(cache.pages, 0x5A), torch.bfloat16)
    sjd.op_kv4_write(fused, k, v, slot, opts=sjd.QkOpts(norm="none"))
    inside = (slots >= 0) & (slots < pages * 64)
    assert len(set(slots[inside])) == inside.sum() > 90
    for got, x, old in zip(sjd.op_kv4_read(cache, everything), (k, v), before):
        old[slots[inside]] = held(_f64(x), "bfloat16")[inside]
        assert np.array_equal(_f64(got), old)
    assert torch.equal(fused.pages, cache.pages)


@pytest.mark.parametrize("name", TYPES)
def test_groups_with_nan_or_infinity_read_as_nan(torch_cuda, name):
    import paper_2505_24791_amd as sjd
    torch = torch_cuda
    rng = np.random.default_rng(5)
    k, v = (_rows(torch, rng, 6, 2, 64, name) for _ in range(2))
    k[1, 0, 3], k[2, 1, 40], v[3, 0, 63], v[4, 1, 0] = float("nan"), float("inf"), float("-inf"), float("nan")
    cache = sjd.Kv4Cache.zeros(1, 2, 64, k.dtype)
    slot = torch.arange(6, dtype=torch.int32, device="cuda")
    sjd.op_kv4_write(cache, k, v, slot)
    for got, x in zip(sjd.op_kv4_read(cache, slot), (k, v)):
        want = held(_f64(x), name)
        assert np.isnan(want).sum() == 64 and np.array_equal(_f64(got), want, equal_nan=True)


@pytest.mark.parametrize("name", TYPES)
@pytest.mark.parametrize("n,H,KV,dim,norm,rot,adjacent,sections", [
    (1, 4, 4, 64, "rms", 64, False, (16, 16)), (77, 6, 2, 128, "layer", 64, True, (10, 22)), (4097, 2, 1, 32, "rms", 32, False, (16,)),
    (10, 8, 8, 256, "none", 0, False, ())])
def test_fused_write_gives_the_bits_of_the_separate_calls(torch_cuda, name, n, H, KV, dim, norm, rot, adjacent, sections):
    import paper_2505_24791_amd as sjd
    torch = torch_cuda
    rng = np.random.default_rng(n + dim)
    qkv = _rows(torch, rng, n, H + 2 * KV, dim, name, 1.0, 3, 1)
    q, k, v = qkv[:, :H], qkv[:, H:H + KV], qkv[:, H + KV:]
    o, ref = _opts(torch, sjd, rng, dim, norm, rot, adjacent, sections)
    pos = torch.from_numpy(rng.integers(0, 5000, (n, max(1, len(sections)))).astype(np.int32)).cuda() if rot else None
    pages = n // 64 + 2
    slot = torch.from_numpy(rng.permutation(pages * 64)[:n].astype(np.int32)).cuda()
    slot[n // 2] = -1
    a, b, c = (sjd.Kv4Cache.zeros(pages, KV, dim, q.dtype) for _ in range(3))
    gq = sjd.op_kv4_write(a, k, v, slot, opts=o, pos=pos, q=q)
    tq, tk = sjd.op_qk_norm_rope(q, k, pos, o)
    sjd.op_kv4_write(b, tk, v, slot)
    assert sjd.op_kv4_write(c, k, v, slot, opts=o, pos=pos) is None
    assert torch.equal(gq, tq) and torch.equal(a.pages, b.pages) and torch.equal(c.pages, b.pages)


# ---- attention ----

def _filled(torch, sjd, rng, name, kv, dim, lens, extra=2, garbage=0xFF):
    """A cache of sequences on shuffled pages, what is not written being garbage; its tables and what it holds."""
    per = [-(-max(n, 0) // 64) for n in lens]
    total = sum(per) + extra
    order = rng.permutation(total)
    table = np.full((len(lens), max(per + [1])), -7, np.int32)
    cache = sjd.Kv4Cache(torch.full((total, kv, 68 * dim), garbage, dtype=torch.uint8, device="cuda"), getattr(torch, name))
    at, keys, values = 0, [], []
    for b, n in enumerate(lens):
        table[b, :per[b]] = order[at:at + per[b]]
        at += per[b]
        k, v = (_rows(torch, rng, n, kv, dim, name) for _ in range(2))
        t = np.arange(n)
        slot = torch.from_numpy((table[b, t // 64] * 64 + t % 64).astype(np.int32)).cuda()
        sjd.op_kv4_write(cache, k, v, slot)
        gk, gv = sjd.op_kv4_read(cache, slot)
        keys.append(_f64(gk))
        values.append(_f64(gv))
    return cache, torch.from_numpy(table).cuda(), torch.tensor(lens, dtype=torch.int32, device="cuda"), keys, values


def _bound(want, mag, big, name, n_keys, dim, top):
    half, f32 = HALF[name], 2.0 ** -24
    scores = 2 * (dim + 8) * f32 * big + 2.0 ** -20          # relative error of a probability: its score's, and the exponential's
    # probabilities are taken relative to the row's largest, 1, in float32: those under its smallest normal number, 2^-126, are zero, which is
    # at most n_keys * 2^-126 * max |v| of the sum (its denominator is at least 1)
    gone = 2.0 ** -126 * top
    return (half * (mag + 2 * np.abs(want)) * 1.01 + (scores + (n_keys + 64) * f32) * (mag + np.abs(want)) + TINY[name] * (1 + 2 * top) + gone)


def _check(torch, got, q, q_start, lens, keys, values, name, **kw):
    got, q64 = _f64(got), _f64(q)
    worst = 0.0
    for b, n_keys in enumerate(lens):
        s = slice(q_start[b], q_start[b + 1])
        if q_start[b] == q_start[b + 1]:
            continue
        want, mag, big = attention(q64[s], keys[b], values[b], n_keys, **kw)
        assert np.isfinite(got[s]).all()
        top = max(1.0, n_keys) * (np.abs(values[b]).max() if n_keys else 0.0)
        err = np.abs(got[s] - want) / np.maximum(_bound(want, mag, big, name, n_keys, q.shape[2], top), 1e-300)
        worst = max(worst, float(err.max()))
        empty = mag.max(-1) == 0
        assert not got[s][empty].any()
    assert worst <= 1.0, worst


@pytest.mark.parametrize("name", TYPES)
def test_large_calls_give_the_bits_of_small_ones(torch_cuda, name):
    """Results of some 50 MB, at odd strides, against the same rows in calls of a thousand; padding between the rows stays."""
    import paper_2505_24791_amd as sjd
    torch = torch_cuda
    rng = np.random.default_rng(8)
    n, H, KV, dim, cut = 10011, 12, 4, 128, 1000
    dt = getattr(torch, name)
    qkv = torch.randn((n, (H + 2 * KV) * dim + 3), dtype=torch.float32, device="cuda").to(dt)
    q, k, v = (qkv[:, 1 + a * dim:1 + b * dim].unflatten(1, (b - a, dim)) for a, b in ((0, H), (H, H + KV), (H + KV, H + 2 * KV)))
    o, _ = _opts(torch, sjd, rng, dim, "layer", 64, False, (16, 16))
    pos = torch.from_numpy(rng.integers(0, 5000, (n, 2)).astype(np.int32)).cuda()
    wide = [torch.full((n, h * dim + 5), 7.0, dtype=dt, device="cuda") for h in (H, KV, H)]
    qo, ko, qw = (w[:, 3:3 + h * dim].unflatten(1, (h, dim)) for w, h in zip(wide, (H, KV, H)))
    slot = torch.from_numpy(rng.permutation((n // 64 + 2) * 64)[:n].astype(np.int32)).cuda()
    sjd.op_qk_norm_rope(q, k, pos, o, q_out=qo, k_out=ko)
    a, b = (sjd.Kv4Cache.zeros(n // 64 + 2, KV, dim, dt) for _ in range(2))
    sjd.op_kv4_write(a, k, v, slot, q=q, pos=pos, opts=o, q_out=qw)
    for i in range(0, n, cut):
        s = slice(i, i + cut)
        gq, gk = sjd.op_qk_norm_rope(q[s], k[s], pos[s], o)
        assert torch.equal(qo[s], gq) and torch.equal(ko[s], gk) and torch.equal(qw[s], gq)
        sjd.op_kv4_write(b, gk, v[s], slot[s])
    for w in wide:
        assert bool((w[:, :3] == 7).all()) and bool((w[:, -2:] == 7).all())
    assert torch.equal(a.pages, b.pages)
    kr, vr = (torch.full((n, KV * dim + 1), 7.0, dtype=dt, device="cuda") for _ in range(2))
    many = slot.repeat(3)
    gk, gv = sjd.op_kv4_read(a, many)                                                  # 62 MB of 16-bit rows
    sjd.op_kv4_read(a, slot, k_out=kr[:, 1:].unflatten(1, (KV, dim)), v_out=vr[:, :-1].unflatten(1, (KV, dim)))
    assert torch.equal(kr[:, 1:].unflatten(1, (KV, dim)), gk[:n]) and bool((kr[:, 0] == 7).all()) and bool((vr[:, -1] == 7).all())
    for j in range(3):
        for i in range(0, n, cut):
            wk, wv = sjd.op_kv4_read(a, slot[i:i + cut])
            at = slice(j * n + i, j * n + min(i + cut, n))
            assert torch.equal(gk[at], wk) and torch.equal(gv[at], wv)


ATTEND = [
    # kv heads, heads, dim, keys of the sequences, new tokens of them, causal, skip, window
    (2, 2, 64, [1, 64, 65, 200], [1, 1, 1, 1], True, 0, 0),
    (1, 1, 32, [49], [1], True, 0, 0),
    (2, 16, 128, [300, 0, 63, 513], [1, 0, 1, 1], True, 0, 0),
    (1, 5, 64, [130, 7, 70], [17, 7, 0], True, 0, 0),
    (3, 6, 32, [100, 90], [33, 90], True, 1, 0),
    (1, 4, 256, [190, 3], [3, 3], True, 0, 50),
    (2, 2, 64, [400, 129], [100, 129], True, 3, 64),
    (1, 2, 128, [77, 640], [9, 2], False, 0, 0),
    (2, 4, 64, [333, 5], [4, 5], False, 2, 100),
    (1, 8, 64, [2, 700], [2, 40], True, 5, 0),
    (2, 8, 128, [500, 70, 65], [60, 70, 1], True, 0, 0),
    (1, 4, 128, [300], [100], True, 2, 33),
    (1, 1, 32, [200, 1000], [200, 129], True, 0, 0),
    (1, 3, 128, [190, 64], [50, 64], False, 1, 0),
]


@pytest.mark.parametrize("name", TYPES)
@pytest.mark.parametrize("case", ATTEND, ids=lambda c: f"{c[1]}of{c[0]}x{c[2]}-{sum(c[4])}new{c[5:]}")
def test_attention(torch_cuda, name, case):
    import paper_2505_24791_amd as sjd
    torch = torch_cuda
    kv, H, dim, lens, new, causal, skip, window = case
    rng = np.random.default_rng(sum(lens) + dim)
    cache, table, kv_len, keys, values = _filled(torch, sjd, rng, name, kv, dim, lens)
    start = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
    q = _rows(torch, rng, int(start[-1]) + 3, H, dim, name, 1.0, 5, 3)
    out = torch.full((q.shape[0], H, dim), 7.0, dtype=q.dtype, device="cuda")
    kw = dict(q_start=torch.from_numpy(start).cuda(), max_q=max(new), max_kv=max(lens), causal=causal, skip_nearest=skip, window=window)
    sjd.op_kv4_attention(cache, q, table, kv_len, out=out, **kw)
    assert (out[int(start[-1]):] == 7.0).all()                            # rows of no sequence
    _check(torch, out, q, start, lens, keys, values, name, causal=causal, skip=skip, window=window)
    # the same bits again, and with bounds that are far too large (the pieces are cut in another way: the same result)
    again = sjd.op_kv4_attention(cache, q, table, kv_len, out=torch.full_like(out, 7.0), **kw)
    assert torch.equal(again, out)
    wide = torch.nn.functional.pad(table, (0, 200), value=2 ** 31 - 1)
    loose = sjd.op_kv4_attention(cache, q, wide, kv_len, out=torch.full_like(out, 7.0), **{**kw, "max_q": 500, "max_kv": None})
    _check(torch, loose, q, start, lens, keys, values, name, causal=causal, skip=skip, window=window)


@pytest.mark.parametrize("name,kv,H,dim,lens", [("bfloat16", 1, 8, 128, [70001]), ("float16", 2, 2, 64, [9000, 1, 20000]),
                                                ("float32", 1, 3, 32, [30000, 500]), ("bfloat16", 1, 1, 256, [12345])])
def test_long_sequences_in_pieces(torch_cuda, name, kv, H, dim, lens):
    import paper_2505_24791_amd as sjd
    torch = torch_cuda
    rng = np.random.default_rng(dim)
    cache, table, kv_len, keys, values = _filled(torch, sjd, rng, name, kv, dim, lens)
    q = _rows(torch, rng, len(lens), H, dim, name, 2.0)
    got = sjd.op_kv4_attention(cache, q, table, kv_len)
    _check(torch, got, q, np.arange(len(lens) + 1), lens, keys, values, name)


def test_scale_and_scores_that_differ_by_much(torch_cuda):
    """A row whose softmax is one key, and one whose scores are large and negative."""
    import paper_2505_24791_amd as sjd
    torch = torch_cuda
    rng = np.random.default_rng(11)
    cache, table, kv_len, keys, values = _filled(torch, sjd, rng, "float32", 1, 64, [500])
    q = _rows(torch, rng, 1, 2, 64, "float32", 30.0)
    got = sjd.op_kv4_attention(cache, q, table, kv_len, scale=2.5)
    _check(torch, got, q, [0, 1], [500], keys, values, "float32", scale=2.5)


def test_bounds_that_are_too_small_and_distances_to_the_ends_of_int32(torch_cuda):
    """Rows beyond max_q stay, the ones before see what they see otherwise; a window or a distance of 2^31 - 1, more new rows than keys."""
    import paper_2505_24791_amd as sjd
    torch = torch_cuda
    rng = np.random.default_rng(31)
    cache, table, kv_len, keys, values = _filled(torch, sjd, rng, "float16", 2, 64, [300, 5])
    start, top = [0, 40, 70], 2 ** 31 - 1
    q = _rows(torch, rng, 70, 4, 64, "float16")
    kw = dict(q_start=torch.tensor(start, dtype=torch.int32, device="cuda"), max_kv=300)
    full = sjd.op_kv4_attention(cache, q, table, kv_len, max_q=40, **kw)
    _check(torch, full, q, start, [300, 5], keys, values, "float16")
    assert not full[40:65].any()                                           # 30 new tokens of which 5 are cached: the first 25 see nothing
    few = sjd.op_kv4_attention(cache, q, table, kv_len, max_q=33, out=torch.full_like(q, 7.0), **kw)
    assert bool((few[33:40] == 7).all())
    _check(torch, torch.cat([few[:33], full[33:40], few[40:]]), q, start, [300, 5], keys, values, "float16")
    wide = sjd.op_kv4_attention(cache, q, table, kv_len, max_q=40, window=top, **kw)
    assert torch.equal(wide, full)
    for skip, window in ((top, 0), (top, top), (301, 1)):
        assert not sjd.op_kv4_attention(cache, q, table, kv_len, max_q=40, skip_nearest=skip, window=window, **kw).any()
    for bad in (dict(window=2 ** 32), dict(skip_nearest=2 ** 32 + 1), dict(max_q=2 ** 32 + 40), dict(max_kv=2 ** 32 + 300)):
        with pytest.raises(sjd.SjdError):
            sjd.op_kv4_attention(cache, q, table, kv_len, **{**dict(max_q=40), **kw, **bad})


def test_pages_that_the_cache_does_not_have_are_not_seen(torch_cuda):
    import paper_2505_24791_amd as sjd
    torch = torch_cuda
    rng = np.random.default_rng(12)
    cache, table, kv_len, keys, values = _filled(torch, sjd, rng, "float16", 2, 64, [400, 100])
    visible = np.ones(400, bool)
    for page, bad in ((1, -1), (3, cache.n_pages), (4, 2 ** 31 - 1), (5, -2 ** 31)):
        table[0, page] = bad
        visible[64 * page:64 * page + 64] = False
    table[1] = -1                                                          # nothing of the second sequence is there
    q = _rows(torch, rng, 2, 4, 64, "float16")
    got = sjd.op_kv4_attention(cache, q, table, kv_len)
    want, mag, big = attention(_f64(q)[:1], keys[0], values[0], 400, visible=visible)
    assert (np.abs(_f64(got)[:1] - want) <= _bound(want, mag, big, "float16", 400, 64, 400 * np.abs(values[0]).max())).all()
    assert not got[1].any()


@pytest.mark.parametrize("name", TYPES)
def test_nan_reaches_the_rows_that_see_it_and_no_other(torch_cuda, name):
    import paper_2505_24791_amd as sjd
    torch = torch_cuda
    rng = np.random.default_rng(13)
    n, L = 20, 150
    cache = sjd.Kv4Cache(torch.full((3, 1, 68 * 64), 0xFF, dtype=torch.uint8, device="cuda"), getattr(torch, name))
    k, v = (_rows(torch, rng, L, 1, 64, name) for _ in range(2))
    v[140, 0, 40] = float("nan")          # seen by the rows at 140 and later: channels 32..63
    k[145, 0, 0] = float("inf")           # all of the rows at 145 and later
    slot = torch.arange(L, dtype=torch.int32, device="cuda")
    sjd.op_kv4_write(cache, k, v, slot)
    q = _rows(torch, rng, n, 2, 64, name)
    table = torch.arange(3, dtype=torch.int32, device="cuda").view(1, 3)
    got = sjd.op_kv4_attention(cache, q, table, torch.tensor([L], dtype=torch.int32, device="cuda"), max_q=n)
    nan = np.isnan(_f64(got))
    first = 140 - (L - n)
    assert not nan[:first].any() and not nan[first:first + 5, :, :32].any()
    assert nan[first:first + 5, :, 32:].all() and nan[first + 5:].all()
    clean_k, clean_v = sjd.op_kv4_read(cache, slot)
    want, mag, big = attention(_f64(q)[:first], _f64(clean_k)[:140], _f64(clean_v)[:140], 140, causal=True)
    # rows before see keys 0 .. 130 + i only: the same as a chunk that ends before the NaN
    assert (np.abs(_f64(got)[:first] - want) <= _bound(want, mag, big, name, L, 64, L * 4.0)).all()
    # a NaN in a query is that row's alone
    q[2, 1, 5] = float("nan")
    again = sjd.op_kv4_attention(cache, q, table, torch.tensor([L], dtype=torch.int32, device="cuda"), max_q=n)
    bad = torch.isnan(again[2, 1])
    assert bad.all()
    again[2, 1] = got[2, 1]
    assert torch.equal(again.view(torch.uint8), got.view(torch.uint8))


def test_cache_beyond_two_gigabytes(torch_cuda):
    """Pages whose bytes lie beyond 2^31: written, read and attended."""
    import paper_2505_24791_amd as sjd
    torch = torch_cuda
    rng = np.random.default_rng(14)
    pages, kv, dim = 8300, 16, 256
    cache = sjd.Kv4Cache(torch.empty((pages, kv, 68 * dim), dtype=torch.uint8, device="cuda"), torch.bfloat16)
    assert cache.pages.numel() > 2 ** 31
    k, v = (_rows(torch, rng, 100, kv, dim, "bfloat16") for _ in range(2))
    table = torch.tensor([[pages - 1, pages - 3]], dtype=torch.int32, device="cuda")
    t = np.arange(100)
    slot = torch.from_numpy((table.cpu().numpy()[0, t // 64] * 64 + t % 64).astype(np.int32)).cuda()
    sjd.op_kv4_write(cache, k, v, slot)
    gk, gv = sjd.op_kv4_read(cache, slot)
    assert np.array_equal(_f64(gk), held(_f64(k), "bfloat16")) and np.array_equal(_f64(gv), held(_f64(v), "bfloat16"))
    q = _rows(torch, rng, 1, 16, dim, "bfloat16")
    got = sjd.op_kv4_attention(cache, q, table, torch.tensor([100], dtype=torch.int32, device="cuda"))
    _check(torch, got, q, [0, 1], [100], [_f64(gk)], [_f64(gv)], "bfloat16")


# ---- together ----

def _layer_step(sjd, s):
    q = sjd.op_kv4_write(s["cache"], s["k"], s["v"], s["slot"], opts=s["opts"], pos=s["pos"], q=s["q"])
    return sjd.op_kv4_attention(s["cache"], q, s["table"], s["kv_len"], max_q=s["max_q"])


def test_a_prompt_and_then_token_by_token(torch_cuda):
    """What a program does with them: a prompt enters the cache and attends it, then single tokens follow; every step against float64 on
    what the cache then holds."""
    import paper_2505_24791_amd as sjd
    torch = torch_cuda
    rng = np.random.default_rng(15)
    B, H, KV, dim, prompt, steps, name = 3, 4, 2, 64, 61, 6, "float16"
    o, ref = _opts(torch, sjd, rng, dim, "rms", 64, False, (16, 16))
    table = torch.from_numpy(rng.permutation(2 * B).astype(np.int32).reshape(B, 2)).cuda()
    cache = sjd.Kv4Cache.zeros(2 * B, KV, dim, torch.float16)
    tnp = table.cpu().numpy()
    slots = lambda t: (tnp[:, t // 64] * 64 + t % 64)                     # [B, len(t)]
    done = 0
    for n in [prompt] + [1] * steps:
        qkv = _rows(torch, rng, B * n, H + 2 * KV, dim, name)
        t = np.arange(done, done + n)
        slot = torch.from_numpy(slots(t).reshape(-1).astype(np.int32)).cuda()
        pos = np.stack([np.tile(t // 8, B), np.tile(t % 8, B)], -1).astype(np.int32)
        done += n
        s = {"cache": cache, "q": qkv[:, :H], "k": qkv[:, H:H + KV], "v": qkv[:, H + KV:], "slot": slot, "opts": o, "table": table, "max_q": n,
             "pos": torch.from_numpy(pos).cuda(), "kv_len": torch.full((B,), done, dtype=torch.int32, device="cuda")}
        got = _layer_step(sjd, s)
        k64 = norm_rotate(_f64(s["k"]), pos, **ref("k"))
        k16 = torch.from_numpy(k64).to(torch.float16).double().numpy()
        every = torch.from_numpy(slots(np.arange(done)).reshape(-1).astype(np.int32)).cuda()
        gk, gv = (_f64(x).reshape(B, done, KV, dim) for x in sjd.op_kv4_read(cache, every))
        assert np.array_equal(gk[:, -n:].reshape(-1, KV, dim), held(k16, name))
        assert np.array_equal(gv[:, -n:].reshape(-1, KV, dim), held(_f64(s["v"]), name))
        q, _ = sjd.op_qk_norm_rope(s["q"], None, s["pos"], o)
        _check(torch, got, q, np.arange(B + 1) * n, [done] * B, gk, gv, name)


def test_captured_step_replays_on_new_inputs(torch_cuda):
    import paper_2505_24791_amd as sjd
    torch = torch_cuda
    rng = np.random.default_rng(16)
    B, H, KV, dim, longest = 2, 4, 1, 128, 3000
    o, _ = _opts(torch, sjd, rng, dim, "rms", 128, True, (32, 32))
    cache, table, kv_len, _, _ = _filled(torch, sjd, rng, "bfloat16", KV, dim, [longest, longest])
    tnp = table.cpu().numpy()

    def inputs(seed):
        r = np.random.default_rng(seed)
        lens = r.integers(1, longest + 1, B)
        qkv = _rows(torch, r, B, H + 2 * KV, dim, "bfloat16")
        return {"q": qkv[:, :H], "k": qkv[:, H:H + KV], "v": qkv[:, H + KV:],
                "slot": torch.from_numpy(np.array([tnp[b, (n - 1) // 64] * 64 + (n - 1) % 64 for b, n in enumerate(lens)], np.int32)).cuda(),
                "pos": torch.from_numpy(np.stack([lens // 50, lens % 50], -1).astype(np.int32)).cuda(),
                "kv_len": torch.from_numpy(lens.astype(np.int32)).cuda()}

    s = {"cache": cache, "opts": o, "table": table, "max_q": 1, **inputs(0)}
    start = cache.pages.clone()
    _layer_step(sjd, s)
    side = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        with torch.cuda.graph(graph, stream=side):
            captured = _layer_step(sjd, s)
    for seed in (1, 2, 3):
        new = inputs(seed)
        cache.pages.copy_(start)
        want = _layer_step(sjd, {**s, **new})
        pages = cache.pages.clone()
        cache.pages.copy_(start)
        for key, t in new.items():
            s[key].copy_(t)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(captured, want) and torch.equal(cache.pages, pages)


def test_calls_on_a_stream_of_their_own(torch_cuda):
    import paper_2505_24791_amd as sjd
    torch = torch_cuda
    rng = np.random.default_rng(17)
    cache, table, kv_len, keys, values = _filled(torch, sjd, rng, "float16", 1, 64, [5000])
    q = _rows(torch, rng, 1, 2, 64, "float16")
    want = sjd.op_kv4_attention(cache, q, table, kv_len)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        got = sjd.op_kv4_attention(cache, q, table, kv_len)
    side.synchronize()
    assert torch.equal(got, want)


def test_no_sequences_and_no_rows(torch_cuda):
    import paper_2505_24791_amd as sjd
    torch = torch_cuda
    cache = sjd.Kv4Cache.zeros(2, 1, 64, torch.float16)
    i32 = lambda *s: torch.zeros(s, dtype=torch.int32, device="cuda")
    q = torch.zeros((0, 2, 64), dtype=torch.float16, device="cuda")
    assert sjd.op_kv4_attention(cache, q, i32(0, 1), i32(0)).shape == (0, 2, 64)
    assert sjd.op_kv4_attention(cache, q, i32(3, 1), i32(3), q_start=i32(4), max_q=0).shape == (0, 2, 64)
    assert sjd.op_kv4_attention(cache, torch.ones((3, 2, 64), dtype=torch.float16, device="cuda"), i32(3, 1), i32(3)).abs().sum() == 0   # no keys
    k = torch.zeros((0, 1, 64), dtype=torch.float16, device="cuda")
    sjd.op_kv4_write(cache, k, k, i32(0))
    assert sjd.op_kv4_read(cache, i32(0))[0].shape == (0, 1, 64)


def test_refused_tensors(torch_cuda):
    import paper_2505_24791_amd as sjd
    torch = torch_cuda
    cache = sjd.Kv4Cache.zeros(2, 2, 64, torch.float16)
    x = torch.zeros((4, 2, 64), dtype=torch.float16, device="cuda")
    i32 = lambda *s: torch.zeros(s, dtype=torch.int32, device="cuda")
    bad = [
        lambda: sjd.op_kv4_write(cache, x.float(), x, i32(4)),                          # another type than the cache's
        lambda: sjd.op_kv4_write(cache, x, x[:3], i32(4)),                              # other rows
        lambda: sjd.op_kv4_write(cache, x, x, i32(4).long()),                           # slots of another type
        lambda: sjd.op_kv4_write(cache, x.transpose(0, 1).contiguous().transpose(0, 1), x, i32(4)),   # heads apart
        lambda: sjd.op_kv4_write(cache, x, x, i32(4), q=x),                             # queries without options
        lambda: sjd.op_kv4_write(cache, x.cpu(), x, i32(4)),
        lambda: sjd.op_kv4_read(cache, i32(4).cpu()),
        lambda: sjd.op_kv4_attention(cache, torch.zeros((1, 3, 64), dtype=torch.float16, device="cuda"), i32(1, 2), i32(1)),   # 3 heads of 2
        lambda: sjd.op_kv4_attention(cache, x, i32(1, 2), i32(1)),                      # four rows of one sequence of one
        lambda: sjd.op_kv4_attention(cache, x[:1], i32(1, 2), i32(1), scale=0.0),
        lambda: sjd.op_kv4_attention(cache, x[:1], i32(1, 2), i32(1), window=-1),
        lambda: sjd.op_qk_norm_rope(x, None, None, sjd.QkOpts(rot_dim=64, axis_pairs=(16, 15), freq=torch.zeros(32, device="cuda"))),
        lambda: sjd.op_qk_norm_rope(x, None, i32(4, 1), sjd.QkOpts(rot_dim=128, axis_pairs=(64,), freq=torch.zeros(64, device="cuda"))),
        lambda: sjd.op_qk_norm_rope(x, None, None, sjd.QkOpts(q_gain=torch.ones(32, device="cuda"))),
        lambda: sjd.op_qk_norm_rope(x[:, :, :60], None, None, sjd.QkOpts()),
        lambda: sjd.QkOpts(norm="batch"),
        lambda: sjd.Kv4Cache(torch.zeros((2, 2, 67), dtype=torch.uint8, device="cuda"), torch.float16),
        lambda: sjd.op_kv4_read(sjd.Kv4Cache.zeros(2, 2, 96, torch.float16), i32(4)),   # a head size that the cache does not have
        lambda: sjd.Kv4Cache.zeros(1, 1, 64, torch.int8),
    ]
    for i, call in enumerate(bad):
        with pytest.raises((sjd.SjdError, AttributeError, TypeError)):
            call()
            pytest.fail(f"call {i} was not refused")

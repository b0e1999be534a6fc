"""Attention over the 4-bit cache where a small mistake would hide in a bound on random sums: keys and queries for which the scores are exact, so
that what is left is a few roundings.  Needs an MI355X.

A key with one channel at 1 has the score that the query holds in that channel, exactly (products and sums of one number and zeros; float32
queries are the sum of their three pieces).  ``half`` is half a step of the rows' type; a probability carries the rounding of its exponent (at
most 2^-19 for exponents below 32) and the exponential's."""
import numpy as np
import pytest

from kv4_reference import attention

pytestmark = [pytest.mark.gpu, pytest.mark.timeout(300)]

HALF = {"float16": 2.0 ** -11, "bfloat16": 2.0 ** -8, "float32": 2.0 ** -24}
TINY = {"float16": 2.0 ** -25, "bfloat16": 0.0, "float32": 0.0}          # half a step of the subnormals
TYPES = list(HALF)


@pytest.fixture(scope="module")
def torch_cuda():
    import torch
    assert torch.cuda.is_available(), "these tests need the GPU"
    return torch


def _f64(t):
    return t.detach().double().cpu().numpy()


def _cached(torch, sjd, name, k, v, rng):
    """A cache that holds k, v [n, kv, dim] (values that the format holds exactly) as one sequence on shuffled pages; its table [1, pages]."""
    n, kv, dim = k.shape
    pages = -(-n // 64)
    table = rng.permutation(pages + 2)[:pages].astype(np.int32)
    dt = getattr(torch, name)
    cache = sjd.Kv4Cache(torch.full((pages + 2, kv, 68 * dim), 0xFF, dtype=torch.uint8, device="cuda"), dt)
    t = np.arange(n)
    slot = torch.from_numpy((table[t // 64] * 64 + t % 64).astype(np.int32)).cuda()
    dk, dv = (torch.from_numpy(x).to(dt).cuda() for x in (k, v))
    sjd.op_kv4_write(cache, dk, dv, slot)
    for got, want in zip(sjd.op_kv4_read(cache, slot), (k, v)):
        assert np.array_equal(_f64(got), want)
    return cache, torch.from_numpy(table).cuda().view(1, -1)


@pytest.mark.parametrize("name", TYPES)
@pytest.mark.parametrize("sink", [0.0, 1.0])
@pytest.mark.parametrize("gap", [14.5, 17.0, 20.0])
def test_the_tail_of_a_softmax_with_one_leading_key(torch_cuda, name, sink, gap):
    """One key ``gap`` nats above 20000 others that hold what the result is made of.  A float16 probability is held to half a step where it is
    2^-21 of the largest and more, below that to 2^-32 of the largest (its subnormals, with probabilities up to 2^7 at the least); every term's error
    counts in full.  Whole sequences a workgroup (many sequences; rows that fill 32-row tiles) and pieces of it."""
    import paper_2505_24791_amd as sjd
    torch = torch_cuda
    rng = np.random.default_rng(40)
    n, dim, first = 20000, 64, 700
    k, v = np.zeros((n, 1, dim)), rng.choice([0.5, 1.0, 1.5], (n, 1, dim))
    k[:, 0, 1], k[first, 0] = 1.0, 0.0
    k[first, 0, 0], v[first] = 1.0, sink
    cache, table = _cached(torch, sjd, name, k, v, rng)
    q = np.zeros((1, 2, dim))
    q[..., 0], q[..., 1] = 8.0, 8.0 - gap
    want, mag, _ = attention(q, k, v, n, causal=False, scale=1.0)
    term = max(HALF[name], 2.0 ** -32 * np.exp(gap)) if name == "float16" else HALF[name]
    sums = (n / 32 + 64) * 2.0 ** -24 + 2.0 ** -18                                    # a lane's sums of a quarter of the keys, scores and exponentials
    bound = (HALF[name] + term + sums) * (mag + np.abs(want)) + TINY[name]
    one = torch.from_numpy(q).to(getattr(torch, name)).cuda()
    for seqs, rows in ((1, 1), (2048, 1), (1, 40), (700, 33)):
        many = one.expand(seqs * rows, 2, dim).contiguous()
        lens = torch.full((seqs,), n, dtype=torch.int32, device="cuda")
        got = sjd.op_kv4_attention(cache, many, table.expand(seqs, -1), lens, max_q=rows, causal=False, scale=1.0)
        assert torch.equal(got, got[:1].expand_as(got)), (seqs, rows)
        worst = (np.abs(_f64(got[:1]) - want) / bound).max()
        assert worst <= 1.0, (seqs, rows, worst)


@pytest.mark.parametrize("name,rows,heads,dim,max_kv,window", [("float32", 131073, 8, 32, None, 50), ("float16", 262200, 8, 64, 20000, 0), ("bfloat16", 131073, 8, 256, None, 70)])
def test_a_prompt_of_more_row_tiles_than_a_grid_counts(torch_cuda, name, rows, heads, dim, max_kv, window):
    """65537 and more tiles of a key head's rows, against the bits of the same rows in calls of 8000.  With a window every row sees the keys before it,
    without one all rows see the same hundred."""
    import paper_2505_24791_amd as sjd
    torch = torch_cuda
    rng = np.random.default_rng(41)
    n, cut = (rows, 8000) if window else (100, 8000)
    g = torch.Generator(device="cuda").manual_seed(41)
    pages = -(-n // 64)
    dt = getattr(torch, name)
    cache = sjd.Kv4Cache.zeros(pages, 1, dim, dt)
    table = torch.from_numpy(rng.permutation(pages).astype(np.int32)).cuda()
    t = torch.arange(n, device="cuda")
    slot = (table[t // 64] * 64 + t % 64).to(torch.int32)
    k, v = (torch.randn((n, 1, dim), generator=g, device="cuda").to(dt) for _ in range(2))
    sjd.op_kv4_write(cache, k, v, slot)
    wide = torch.nn.functional.pad(table, (0, 400)).view(1, -1)
    q = torch.randn((rows, heads, dim), generator=g, device="cuda").to(dt)
    i32 = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")
    kw = dict(causal=bool(window), window=window)
    got = sjd.op_kv4_attention(cache, q, wide, i32(n), q_start=i32(0, rows), max_q=rows, max_kv=max_kv or n, **kw)
    for i in range(0, rows, cut):
        part = q[i:i + cut]
        m = len(part)
        kv_len = i + m if window else n
        want = sjd.op_kv4_attention(cache, part, wide, i32(kv_len), max_q=m, max_kv=max_kv or n, **kw)
        assert torch.equal(got[i:i + m], want), i
    assert not torch.equal(got[:8000], got[-8000:])


@pytest.mark.parametrize("name", TYPES)
@pytest.mark.parametrize("n,dim,every", [(64 * 40 + 17, 64, 1), (30017, 128, 9)])
def test_every_key_counts_once(torch_cuda, name, n, dim, every):
    """Two equal keys on either side of a border (of a page, of a subtile of 16, the first and last of all) with a query that only they answer to: the
    result is the mean of their values, and a key that is dropped or taken twice moves it by a sixth of their difference and more, 1/12 at the least.  Keys are
    +-1 in every channel, so that the two have the score 2 dim and no other comes within 45 of it.

    Bound: the two probabilities are the same number.  A sum of the matrix unit is not always the nearest float32 (what is 2^-65 below a sum can take it
    a whole step down), so a term counts one step, 2^-23, of a partial sum of at most 3: six of them (three pieces of two keys), four waves, the
    pieces' join, the reciprocal and the product are below 16, together 3 * 2^-19.  A mean is a multiple of 1/4 below 4, which 16 bits hold, so that rounding
    to them takes the result back to it, or, where it is zero, leaves it within the same bound."""
    import paper_2505_24791_amd as sjd
    torch = torch_cuda
    rng = np.random.default_rng(42 + dim)
    kv, group = 2, 3
    dt = getattr(torch, name)
    k = rng.choice([-1.0, 1.0], (n, kv, dim))
    v = rng.choice([-3.0, -2.0, -1.5, -1.0, -0.5, 0.5, 1.0, 1.5, 2.0, 3.0], (n, kv, dim))
    pairs = [(0, n - 1)]
    for p in range(1, n // 64, every):
        pairs += [(64 * p - 1, 64 * p), (64 * p + 15, 64 * p + 16), (64 * p + 31, 64 * p + 47)]
    a, b = np.array(pairs).T
    assert len(set(a) | set(b)) == 2 * len(pairs)
    k[b] = k[a]
    other = np.einsum("phd,nhd->phn", k[a], k, optimize=True) * 2.0
    for i, x in enumerate(pairs):
        other[i][:, x] = -np.inf
    assert other.max() <= 2 * dim - 45
    cache, table = _cached(torch, sjd, name, k, v, rng)
    q = torch.from_numpy(2.0 * np.repeat(k[a], group, 1)).to(dt).cuda()
    want = torch.from_numpy(np.repeat((v[a] + v[b]) / 2, group, 1)).cuda()
    lens = lambda s: torch.full((s,), n, dtype=torch.int32, device="cuda")
    m = len(pairs)
    copies = -(-32768 // (m * group * kv)) + 1                                       # rows for more workgroups than are wanted: no pieces
    runs = {"single tokens, pieces": lambda: (q, m, 1, None), "a chunk, pieces": lambda: (q, 1, m, None), "a chunk, pieces of 32-row tiles": lambda: (q, 1, m, n + 30000),
            "single tokens": lambda: (q.repeat(-(-2048 // (m * kv)), 1, 1), None, 1, None), "a chunk": lambda: (q.repeat(copies, 1, 1), 1, None, None),
            "a chunk, 32-row tiles": lambda: (q.repeat(copies, 1, 1), 1, None, n + 30000)}
    for what, make in runs.items():
        rows, seqs, each, most = make()
        seqs, each = seqs or len(rows), each or len(rows)
        got = sjd.op_kv4_attention(cache, rows, torch.nn.functional.pad(table, (0, 500)).expand(seqs, -1), lens(seqs), max_q=each, max_kv=most or n, causal=False, scale=1.0)
        ref = want.repeat(len(rows) // m, 1, 1)
        assert float((got.double() - ref).abs().max()) <= 3 * 2.0 ** -19, what


def _pieces(x, n):
    """The first n bfloat16 pieces of float32 values, summed."""
    import torch
    left, total = torch.from_numpy(np.asarray(x, np.float64)), 0.0
    for _ in range(n):
        p = left.float().to(torch.bfloat16).double()
        total, left = total + p, left - p
    return total.numpy()


def test_float32_queries_keep_24_bits(torch_cuda):
    """Eight keys of one channel each, scores between 4 and 8 that hold all bits of float32.  A probability is good to 2^-21: the
    exponent's one rounding below 8 (2^-22 ln 2), the scale's (2^-25 of 4), the exponential's (2^-23); then three times 8 sums, the waves' and the
    quotient (40 in all).  With two pieces of the queries the same bound fails."""
    import paper_2505_24791_amd as sjd
    torch = torch_cuda
    rng = np.random.default_rng(43)
    n, dim, rows, H = 8, 32, 64, 4
    k, v = np.zeros((n, 1, dim)), rng.choice([-3.0, -2.0, -1.0, -0.5, 0.5, 1.0, 2.0, 3.0], (n, 1, dim))
    k[np.arange(n), 0, np.arange(n)] = 1.0
    cache, table = _cached(torch, sjd, "float32", k, v, rng)
    q = np.zeros((rows, H, dim))
    q[..., :n] = rng.uniform(4, 8, (rows, H, n)).astype(np.float32)
    want, mag, _ = attention(q, k, v, n, causal=False, scale=1.0)
    bound = (2.0 ** -21 + 40 * 2.0 ** -24) * (mag + np.abs(want))
    planted, _, _ = attention(_pieces(q, 2), k, v, n, causal=False, scale=1.0)
    assert (np.abs(planted - want) / bound).max() > 2
    lens = torch.tensor([n], dtype=torch.int32, device="cuda")
    got = sjd.op_kv4_attention(cache, torch.from_numpy(q).float().cuda(), table, lens, max_q=rows, causal=False, scale=1.0)
    assert (np.abs(_f64(got) - want) / bound).max() <= 1


def test_float32_probabilities_keep_24_bits(torch_cuda):
    """Two keys that count, four pages apart so that one wave has both, the second 1 to 5 nats above the first: its probability then is any number
    between 2 and 2^8 (the reference does not move for it).  The same bound as above, with two terms to sum; with two pieces of
    the probability, against the whole one in the denominator, it fails."""
    import paper_2505_24791_amd as sjd
    torch = torch_cuda
    rng = np.random.default_rng(44)
    n, dim, rows = 257, 32, 2048
    k, v = np.zeros((n, 1, dim)), rng.choice([-3.0, -2.0, -1.0, -0.5, 0.5, 1.0, 2.0, 3.0], (n, 1, dim))
    k[:, 0, 31] = 1.0
    for t, c in ((0, 0), (256, 1)):
        k[t, 0, 31], k[t, 0, c] = 0.0, 1.0
    cache, table = _cached(torch, sjd, "float32", k, v, rng)
    q = np.zeros((rows, 1, dim))
    q[..., 0] = rng.uniform(0.5, 2, (rows, 1)).astype(np.float32)
    q[..., 1] = (q[..., 0] + rng.uniform(1, 5, (rows, 1))).astype(np.float32)
    q[..., 31] = -1000.0
    p = np.exp(q[..., 1] - q[..., 0])[..., None]
    form = lambda held: (v[0] + held * v[256]) / (1 + p)
    want, mag = form(p), (np.abs(v[0]) + p * np.abs(v[256])) / (1 + p)
    bound = (2.0 ** -21 + 12 * 2.0 ** -24) * (mag + np.abs(want))
    assert (np.abs(form(_pieces(p, 2)) - want) / bound).max() > 2
    lens = torch.full((rows,), n, dtype=torch.int32, device="cuda")
    got = sjd.op_kv4_attention(cache, torch.from_numpy(q).float().cuda(), table.expand(rows, -1), lens, scale=1.0)
    assert (np.abs(_f64(got) - want) / bound).max() <= 1


def _grouped(rng, n, kv, dim, exponents):
    """Values of the format: every group of 32 with its largest at 4 or 6 times 2^exponent; exponents [n, kv, dim / 32], None where all are zero."""
    x = rng.choice([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], (n, kv, dim // 32, 32)) * rng.choice([-1, 1], (n, kv, dim // 32, 32))
    x[..., 0] = rng.choice([4.0, 6.0], x.shape[:-1])
    x = np.ldexp(rng.permuted(x, axis=-1), exponents[..., None])
    zero = rng.random(exponents.shape) < 0.1
    x[zero] = 0.0
    return x.reshape(n, kv, dim)


RANGE = {"float16": (-23, 13), "bfloat16": (-125, 125), "float32": (-125, 125)}


@pytest.mark.parametrize("name", TYPES)
@pytest.mark.parametrize("dim", [32, 64, 128, 256])
def test_values_of_every_scale_as_one_row_sees_them(torch_cuda, name, dim):
    """Each group of a key and a value at a power of two of its own, over all of the type's range (values below 2^96), subnormals of float16 among
    them, next to groups of zeros.  A row that sees one key gives its value back: exactly, in 16 bits."""
    import paper_2505_24791_amd as sjd
    torch = torch_cuda
    rng = np.random.default_rng(45 + dim)
    n, kv, H = 203, 2, 4
    lo, hi = RANGE[name]
    ek, ev = rng.integers(lo, hi + 1, (n, kv, dim // 32)), rng.integers(lo, min(hi, 92) + 1, (n, kv, dim // 32))
    ek[:5], ev[:5], ev[5:9] = lo, lo, min(hi, 92)
    k, v = _grouped(rng, n, kv, dim, ek), _grouped(rng, n, kv, dim, ev)
    cache, table = _cached(torch, sjd, name, k, v, rng)
    lens = torch.tensor([n], dtype=torch.int32, device="cuda")
    # queries against which the key that a row sees has a score of some ten
    top = 14 if name == "float16" else 120
    q = rng.standard_normal((n, kv, dim // 32, 32)) * np.exp2(np.clip(-ek, -top, top - 3))[..., None] / np.sqrt(dim)
    want = np.repeat(v, H // kv, 1)
    for scaled in (0.0, 1.0):
        dq = torch.from_numpy(np.repeat(scaled * q.reshape(n, kv, dim), H // kv, 1)).to(getattr(torch, name)).cuda()
        got = _f64(sjd.op_kv4_attention(cache, dq, table, lens, max_q=n, window=1, scale=1.0))
        if name == "float32":
            assert (np.abs(got - want) <= 2.0 ** -21 * np.abs(want)).all()
        else:
            assert np.array_equal(got, want)
    alone = torch.arange(1, dtype=torch.int32, device="cuda")
    got = sjd.op_kv4_attention(cache, dq[:1], table, alone + 1, scale=1.0)
    assert (np.abs(_f64(got) - want[:1]) <= (2.0 ** -21 if name == "float32" else 0.0) * np.abs(want[:1])).all()


@pytest.mark.parametrize("name", TYPES)
@pytest.mark.parametrize("dim", [32, 64, 128, 256])
@pytest.mark.parametrize("small", [True, False])
def test_scores_of_keys_of_every_scale(torch_cuda, name, dim, small):
    """Groups of channels whose keys lie at far powers of two, with queries at the inverse ones, so that all of them count in the scores."""
    import paper_2505_24791_amd as sjd
    torch = torch_cuda
    rng = np.random.default_rng(46 + dim)
    n, kv, H, rows = 150, 2, 4, 9
    # key exponents, what queries and keys multiply to, and the scale that takes it back
    lo, hi, product = {"float16": ((-23, -9, -9), (-9, 13, 0)), "bfloat16": ((-125, 0, -60), (0, 125, 60)), "float32": ((-125, 0, -60), (0, 125, 60))}[name][0 if small else 1]
    e = rng.integers(lo, hi + 1, (1, kv, dim // 32))
    e[..., 0] = lo if small else hi
    vlo, vhi = RANGE[name]
    ev = np.clip(rng.integers(vlo, min(vhi, 90) + 1, (1, kv, dim // 32)) + rng.integers(-2, 3, (n, kv, dim // 32)), vlo, vhi)
    k = _grouped(rng, n, kv, dim, np.clip(e + rng.integers(-1, 2, (n, kv, dim // 32)), *RANGE[name]))
    v = _grouped(rng, n, kv, dim, ev)
    cache, table = _cached(torch, sjd, name, k, v, rng)
    q = rng.standard_normal((rows, kv, dim // 32, 32)) * np.exp2(product - e)[..., None]
    dq = torch.from_numpy(np.repeat(q.reshape(rows, kv, dim), H // kv, 1)).to(getattr(torch, name)).cuda()
    q64 = _f64(dq)
    scale = 2.0 ** -product / 2.5 * dim ** -0.5
    scale = float(np.float32(scale))
    want, mag, big = attention(q64, k, v, n, causal=False, scale=scale)
    assert 1 < big < 60
    # a score's sums over the channels, the waves' and keys' sums, probabilities and result rounded once; float16 probabilities below 2^-21 of the largest, and
    # results among its subnormals
    f32, half = 2.0 ** -24, HALF[name]
    scores = 2 * (dim + 8) * f32 * big + 2.0 ** -20
    tail = n * 2.0 ** -32 * np.abs(v).max((0, 2))[None, :, None].repeat(H // kv, 1) if name == "float16" else 0.0
    bound = (2 * half + scores + (n + 64) * f32) * (mag + np.abs(want)) + TINY[name] + tail
    lens = torch.tensor([n], dtype=torch.int32, device="cuda")
    got = _f64(sjd.op_kv4_attention(cache, dq, table, lens, max_q=rows, causal=False, scale=scale))
    assert (np.abs(got - want) <= bound).all(), (np.abs(got - want) / bound).max()


def test_calls_do_not_wait_for_another_stream(torch_cuda):
    """All four calls on a stream of their own end, with the results of the current one, while a long row of products still runs on the default stream: they are
    on the stream that is current, and on no other."""
    import paper_2505_24791_amd as sjd
    torch = torch_cuda
    rng = np.random.default_rng(47)
    n, H, dim = 5000, 2, 64
    k, v = (torch.from_numpy(rng.standard_normal((n, 1, dim))).half().cuda() for _ in range(2))
    q = torch.from_numpy(rng.standard_normal((n, H, dim))).half().cuda()
    pages = -(-n // 64)
    i32 = lambda x: torch.as_tensor(x, dtype=torch.int32, device="cuda")
    slot, table, lens, pos = i32(np.arange(n)), i32(np.arange(pages)).view(1, -1), i32([n]), i32(np.arange(n)).view(-1, 1)
    freq = torch.rand(32, device="cuda")
    opts = sjd.QkOpts(rot_dim=64, axis_pairs=(32,), freq=freq)
    busy = torch.randn((8192, 8192), device="cuda").half()

    def calls():
        cache = sjd.Kv4Cache(torch.zeros((pages, 1, 68 * dim), dtype=torch.uint8, device="cuda"), torch.float16)
        turned, _ = sjd.op_qk_norm_rope(q, None, pos, opts)
        sjd.op_kv4_write(cache, k, v, slot)
        held = sjd.op_kv4_read(cache, slot)
        fused = sjd.op_kv4_write(cache, k, v, slot, opts=opts, pos=pos, q=q)
        return [turned, *held, fused, sjd.op_kv4_attention(cache, fused[:1], table, lens), cache.pages]

    want = calls()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        calls()                                    # memory of this stream's own, for the run below
    torch.cuda.synchronize()
    out = torch.empty_like(busy)
    done = torch.cuda.Event()
    for _ in range(300):
        torch.mm(busy, busy, out=out)
    done.record()
    with torch.cuda.stream(side):
        got = calls()
        same = [torch.equal(a, b) for a, b in zip(got, want)]
    side.synchronize()
    early = not done.query()
    torch.cuda.synchronize()
    assert all(same) and early


@pytest.mark.parametrize("name", TYPES)
def test_results_in_the_place_of_the_queries(torch_cuda, name):
    """Single tokens and a chunk, in pieces and whole, one and several tiles: the bits of a call with a result of its own."""
    import paper_2505_24791_amd as sjd
    torch = torch_cuda
    rng = np.random.default_rng(48)
    n, dim, H = 3000, 64, 6
    k, v = (rng.choice([-3.0, -1.0, 0.5, 2.0], (n, 2, dim)) for _ in range(2))
    cache, table = _cached(torch, sjd, name, k, v, rng)
    for seqs, rows in ((3, 1), (1100, 1), (1, 100), (2, 1500)):
        lens = torch.full((seqs,), n, dtype=torch.int32, device="cuda")
        base = torch.from_numpy(rng.standard_normal((seqs * rows, H * dim + 5))).to(getattr(torch, name)).cuda()
        q = base[:, 3:3 + H * dim].unflatten(1, (H, dim))
        want = sjd.op_kv4_attention(cache, q.clone(), table.expand(seqs, -1), lens, max_q=rows)
        pad = base[:, :3].clone()
        assert sjd.op_kv4_attention(cache, q, table.expand(seqs, -1), lens, max_q=rows, out=q) is q
        assert torch.equal(q, want) and torch.equal(base[:, :3], pad)


def test_a_gain_whose_storage_is_replaced(torch_cuda):
    """``param.data = ...`` between two calls with the same options: the second reads the new values, in place of memory that is anyone's by then."""
    import paper_2505_24791_amd as sjd
    torch = torch_cuda
    gain = torch.nn.Parameter(torch.full((64,), 2.0, device="cuda"))
    opts = sjd.QkOpts(q_gain=gain, eps=0.0)
    q = torch.ones((5, 3, 64), device="cuda")
    assert bool((sjd.op_qk_norm_rope(q, None, None, opts)[0] == 2).all())
    gain.data = torch.full((64,), 3.0, device="cuda")
    other = [torch.full((64,), 7.0, device="cuda") for _ in range(8)]              # takes the old one's place
    assert bool((sjd.op_qk_norm_rope(q, None, None, opts)[0] == 3).all()) and len(other) == 8
    gain.data = gain.data.cpu()
    with pytest.raises(sjd.SjdError):
        sjd.op_qk_norm_rope(q, None, None, opts)


def test_two_captured_graphs_replayed_at_once(torch_cuda):
    """Two graphs over one cache, each with pieces to join, replayed side by side on two streams: a workspace belongs to one of them."""
    import paper_2505_24791_amd as sjd
    torch = torch_cuda
    rng = np.random.default_rng(49)
    n, dim, H = 20000, 128, 8
    k, v = (rng.choice([-3.0, -1.0, 0.5, 2.0], (n, 2, dim)) for _ in range(2))
    cache, table = _cached(torch, sjd, "bfloat16", k, v, rng)
    lens = torch.tensor([n], dtype=torch.int32, device="cuda")
    qs = [torch.from_numpy(rng.standard_normal((1, H, dim))).bfloat16().cuda() for _ in range(2)]
    sides, graphs, outs = [torch.cuda.Stream() for _ in qs], [], []
    sjd.op_kv4_attention(cache, qs[0], table, lens)
    torch.cuda.synchronize()
    for q, side in zip(qs, sides):
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1], stream=side):
            outs.append(sjd.op_kv4_attention(cache, q, table, lens))
    for seed in range(4):
        for q in qs:
            q.copy_(torch.from_numpy(rng.standard_normal((1, H, dim))))
        want = [sjd.op_kv4_attention(cache, q, table, lens) for q in qs]
        torch.cuda.synchronize()
        for _ in range(20):
            for graph, side in zip(graphs, sides):
                with torch.cuda.stream(side):
                    graph.replay()
        torch.cuda.synchronize()
        for got, w in zip(outs, want):
            assert torch.equal(got, w), seed

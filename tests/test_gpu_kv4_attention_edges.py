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

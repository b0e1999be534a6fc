"""The attention-side operators that are timed: queries and keys normed for each head and rotated by their positions,
a key/value cache held in 4 bits that is written and read back, and attention over that cache.

Cache format (``sjd_kv4`` in ``include/sjd.h``): pages of 64 tokens; 32 consecutive channels of one token and head share a
power of two s = 2^e, and each is held as one of 0, 1/2, 1, 3/2, 2, 3, 4, 6 times s with a sign.  e is the smallest exponent
with max |x| <= 7 s, within what the type of the rows allows; ties go to the level with an even index.
"""
import math

import torch

own = False

PAGE = 64
_TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
_EXPONENTS = {"f32": (-125, 125), "bf16": (-125, 125), "f16": (-23, 13)}


# ------------------------------------------------------------------------------------------------ cases

def _rope(name, rows, heads, kv_heads, dim, dtype, norm, axes, rot, pairing, far=1):
    return {"name": name, "op": "rope", "rows": rows, "heads": heads, "kv_heads": kv_heads, "dim": dim, "dtype": dtype, "norm": norm,
            "axes": axes, "rot": rot, "pairing": pairing, "far": far}


def _write(name, rows, heads, kv_heads, dim, dtype, norm, axes, rot, pairing, order, holes=0, far=1):
    return {"name": name, "op": "write", "rows": rows, "heads": heads, "kv_heads": kv_heads, "dim": dim, "dtype": dtype, "norm": norm,
            "axes": axes, "rot": rot, "pairing": pairing, "far": far, "order": order, "holes": holes}


def _read(name, rows, kv_heads, dim, dtype, order):
    return {"name": name, "op": "read", "rows": rows, "kv_heads": kv_heads, "dim": dim, "dtype": dtype, "order": order}


def _attend(name, seqs, heads, kv_heads, dim, dtype, shortest, longest, new, ragged_new=0, causal=1, skip=0, window=0):
    return {"name": name, "op": "attend", "seqs": seqs, "heads": heads, "kv_heads": kv_heads, "dim": dim, "dtype": dtype,
            "shortest": shortest, "longest": longest, "new": new, "ragged_new": ragged_new, "causal": causal, "skip": skip,
            "window": window}


def listed():
    return [
        # one token of each of 32 sequences in the middle of sampling 32x32 patches (row, column): the call costs more than the work
        _rope("rotate a step", 32, 16, 16, 64, "bf16", "rms", 2, 64, 0),
        # the whole-sequence pass of 32 samples of 1024 patches, width 1024
        _rope("rotate images", 32768, 16, 16, 64, "f16", "rms", 2, 64, 0),
        # a clip of 17 frames of 45x13 patches (time, row, column): shared key heads, adjacent pairs, an odd number of rows
        _rope("rotate video", 9945, 32, 8, 128, "bf16", "layer", 3, 128, 1, far=7),
        # one token of 256 samples enters the cache: queries and keys normed and rotated in the same call, a few rows of padding
        _write("cache a step", 256, 12, 12, 64, "f16", "rms", 2, 64, 0, "scattered", holes=5),
        # whole prompts enter the cache: 32 samples of 1024 tokens, width 1024
        _write("cache prompts", 32768, 16, 16, 64, "bf16", "rms", 2, 64, 0, "pages"),
        # keys and values of a small float32 model as they are, far positions rotated in part
        _write("cache small float32", 3001, 8, 4, 32, "f32", "none", 1, 16, 0, "pages", far=100000),
        # some cached tokens handed back to a 16-bit path, from all over the cache
        _read("read back some", 1000, 8, 128, "f16", "scattered"),
        # a whole cache handed back
        _read("read back all", 40000, 16, 64, "bf16", "pages"),
        # single-token attention of a small float32 model: 4 samples, 49 tokens
        _attend("attend small float32", 4, 4, 4, 32, "f32", 49, 49, 1),
        # single-token attention of a batch of 256 in the middle of sampling, every sequence at its own length
        _attend("attend a step", 256, 12, 12, 64, "f16", 1, 1024, 1),
        # single-token attention over long contexts with shared key heads
        _attend("attend long", 16, 32, 8, 128, "bf16", 20000, 65536, 1),
        # a chunk of new tokens of a few sequences against what is cached of them and their own; the nearest position is masked
        # (tokens of some sequences are their first: a row without a key among them)
        _attend("attend a chunk", 8, 16, 16, 64, "f16", 500, 4000, 500, ragged_new=1, skip=1),
    ]


def _spread(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _some_rope(rng, most):
    dim = rng.choice((32, 64, 64, 128, 128, 256))
    kv = rng.choice((1, 2, 4, 8, 12, 16))
    heads = kv * rng.choice((1, 1, 2, 3, 4, 8))
    rot = rng.choice((dim, dim, dim // 2))
    axes = rng.choice((1, 2, 3))
    return {"rows": _spread(rng, 1, max(1, min(40000, most // ((heads + kv) * dim)))), "heads": heads, "kv_heads": kv, "dim": dim,
            "dtype": rng.choice(("f32", "bf16", "f16")), "norm": rng.choice(("none", "rms", "layer")), "axes": axes, "rot": rot,
            "pairing": rng.choice((0, 1)), "far": rng.choice((1, 50, 100000))}


def draw(rng):
    op = rng.choice(("rope", "write", "read", "attend", "attend"))
    if op == "rope":
        return {"op": "rope", **_some_rope(rng, 60_000_000)}
    if op == "write":
        c = _some_rope(rng, 40_000_000)
        return {"op": "write", **c, "order": rng.choice(("pages", "scattered")), "holes": rng.choice((0, 1, 3))}
    if op == "read":
        dim, kv = rng.choice((32, 64, 128, 256)), rng.choice((1, 2, 4, 8, 12, 16))
        return {"op": "read", "rows": _spread(rng, 1, min(60000, 40_000_000 // (dim * kv))), "kv_heads": kv, "dim": dim,
                "dtype": rng.choice(("f32", "bf16", "f16")), "order": rng.choice(("pages", "scattered"))}
    dim, kv = rng.choice((32, 64, 64, 128, 128, 256)), rng.choice((1, 2, 4, 8, 12, 16))
    heads = kv * rng.choice((1, 1, 2, 4, 8))
    dtype = rng.choice(("f32", "bf16", "bf16", "f16", "f16"))
    seqs = _spread(rng, 1, 256)
    new = rng.choice((1, 1, 1, rng.randint(2, 9), _spread(rng, 10, 700)))
    # within the largest listed cases: cached values, scores
    most = min(500_000_000 // (seqs * kv * dim), 400_000_000 // (seqs * heads * new), 60000)
    longest = _spread(rng, max(1, min(new, most)), max(1, most))
    return {"op": "attend", "seqs": seqs, "heads": heads, "kv_heads": kv, "dim": dim, "dtype": dtype,
            "shortest": max(1, int(longest * rng.choice((1.0, 0.5, 0.01)))), "longest": longest, "new": min(new, longest),
            "ragged_new": rng.choice((0, 1)), "causal": rng.choice((1, 1, 1, 0)), "skip": rng.choice((0, 0, 1, 3)),
            "window": rng.choice((0, 0, 0, 100))}


# ------------------------------------------------------------------------------------------------ what the format means

def _power(e):
    """2^e in float32 for exponents down to -127 (zero there)."""
    return ((e.to(torch.int32) + 127) << 23).view(torch.float32)


def _codes(x, dtype):
    """x [..., dim] -> the 4-bit codes of every value (uint8) and the exponents of every group of 32."""
    lo, hi = _EXPONENTS[dtype]
    x = x.float()
    g = x.reshape(*x.shape[:-1], -1, 32)
    m, e = torch.frexp(g.abs().amax(-1))                       # 2^(e-1) <= max < 2^e
    e = (e - 3 + (m > 0.875)).clamp(lo, hi)
    e = torch.where(m == 0, torch.full_like(e, lo), e)
    a = g.abs() * _power(-e).unsqueeze(-1)
    c = ((a > 0.25).byte() + (a >= 0.75) + (a > 1.25) + (a >= 1.75) + (a > 2.5) + (a >= 3.5) + (a > 5.0))
    c = (c + 8 * torch.signbit(g).byte()).to(torch.uint8)
    return c.reshape(x.shape), e


def _values(c, e):
    """The float32 values of codes [..., dim] and exponents [..., dim / 32]."""
    m = (c & 7).to(torch.int32)
    # levels 0, 1/2, 1, 3/2, 2, 3, 4, 6: a two-bit exponent and one bit below the leading one
    v = torch.where(m < 2, 0.5 * m, (1.0 + 0.5 * (m & 1)) * _power((m >> 1) - 1))
    v = torch.where((c & 8) != 0, -v, v)
    g = v.reshape(*v.shape[:-1], -1, 32)
    return (g * _power(e).unsqueeze(-1)).reshape(v.shape)


# Where the values of a token are in the 68 dim bytes that a page takes for each head, NG = dim / 32 groups:
#   keys      byte offset * dim / 2 + c / 2, the low half of a byte first
#   values    32 dim + (offset / 16) * 8 dim + (((offset % 16 / 4) * 16 + c % 32 / 2) * 4 + offset % 4) * NG + c / 32
#   key exponents    64 dim + ((offset % 16) * NG + g) * 4 + offset / 16          (exponent + 127)
#   value exponents  66 dim + (offset % 16 / 4) * 16 NG + (offset / 16) * 4 NG + (offset % 4) * NG + g

def _pages_of(k, v, dtype):
    """k, v [pages, kv_heads, 64, dim] -> the pages' bytes [pages, kv_heads, 68 dim]."""
    P, H, _, dim = k.shape
    ng = dim // 32
    kc, ke = _codes(k, dtype)
    vc, ve = _codes(v, dtype)
    kb = (kc[..., 0::2] | (kc[..., 1::2] << 4)).reshape(P, H, 32 * dim)
    vb = (vc[..., 0::2] | (vc[..., 1::2] << 4)).reshape(P, H, 4, 4, 4, ng, 16)          # subtile, four, token, group, pair
    vb = vb.permute(0, 1, 2, 3, 6, 4, 5).reshape(P, H, 32 * dim)
    ks = (ke + 127).to(torch.uint8).reshape(P, H, 4, 16, ng).permute(0, 1, 3, 4, 2).reshape(P, H, 2 * dim)
    vs = (ve + 127).to(torch.uint8).reshape(P, H, 4, 4, 4, ng).permute(0, 1, 3, 2, 4, 5).reshape(P, H, 2 * dim)
    return torch.cat((kb, vb, ks, vs), -1)


def _of_pages(pages, dim):
    """The float32 keys and values [pages, kv_heads, 64, dim] of pages [pages, kv_heads, 68 dim]."""
    P, H, _ = pages.shape
    ng = dim // 32
    kb = pages[..., :32 * dim].reshape(P, H, PAGE, dim // 2)
    vb = pages[..., 32 * dim:64 * dim].reshape(P, H, 4, 4, 16, 4, ng).permute(0, 1, 2, 3, 5, 6, 4).reshape(P, H, PAGE, dim // 2)
    ks = pages[..., 64 * dim:66 * dim].reshape(P, H, 16, ng, 4).permute(0, 1, 4, 2, 3).reshape(P, H, PAGE, ng)
    vs = pages[..., 66 * dim:].reshape(P, H, 4, 4, 4, ng).permute(0, 1, 3, 2, 4, 5).reshape(P, H, PAGE, ng)
    split = lambda b: torch.stack((b & 15, b >> 4), -1).reshape(*b.shape[:-1], dim)  # noqa: E731
    return _values(split(kb), ks.to(torch.int32) - 127), _values(split(vb), vs.to(torch.int32) - 127)


def _token_bytes(off, dim):
    """Where the bytes of a token at page offset off [n] are: keys, values [n, dim / 2], their exponents [n, dim / 32]."""
    ng = dim // 32
    off = off.unsqueeze(-1)
    pair = torch.arange(dim // 2, device=off.device)
    g = torch.arange(ng, device=off.device)
    kb = off * (dim // 2) + pair
    vb = 32 * dim + (off // 16) * 8 * dim + (((off % 16 // 4) * 16 + pair % 16) * 4 + off % 4) * ng + pair // 16
    ks = 64 * dim + ((off % 16) * ng + g) * 4 + off // 16
    vs = 66 * dim + (off % 16 // 4) * 16 * ng + (off // 16) * 4 * ng + (off % 4) * ng + g
    return torch.cat((kb, vb, ks, vs), -1)


# ------------------------------------------------------------------------------------------------ inputs

def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _slots(n, order, g):
    """n different token slots of a cache that is a quarter larger: the tokens of whole pages (which are anywhere), or any."""
    pages = -(-n // PAGE) + max(1, n // (4 * PAGE))
    if order == "scattered":
        s = torch.randperm(pages * PAGE, generator=g, device="cuda")[:n]
    else:
        s = (torch.randperm(pages, generator=g, device="cuda").unsqueeze(1) * PAGE + torch.arange(PAGE, device="cuda")).reshape(-1)[:n]
    return s.to(torch.int32).contiguous(), pages


def _normed_rows(case, g):
    """Rows of a q/k/v projection, gains and shifts of the norms, positions and frequencies."""
    n, H, KV, dim, dtype = case["rows"], case["heads"], case["kv_heads"], case["dim"], _TYPES[case["dtype"]]
    qkv = torch.randn((n, (H + 2 * KV) * dim), generator=g, device="cuda").to(dtype)
    rand = lambda *s: torch.randn(s, generator=g, device="cuda")  # noqa: E731
    pairs, axes = case["rot"] // 2, case["axes"]
    sections = [pairs // axes] * (axes - 1)
    sections.append(pairs - sum(sections))
    # each axis has its own geometric run of frequencies
    freq = torch.cat([10000.0 ** (-torch.arange(p, dtype=torch.float64) / p) for p in sections]).float().cuda()
    side = max(2, int(round(min(n, 1024) ** (1.0 / axes))))
    at = torch.arange(n, device="cuda")
    pos = torch.stack([(at // side ** (axes - 1 - a)) % side for a in range(axes)], -1) * case["far"]
    s = {"q": qkv[:, :H * dim].view(n, H, dim), "k": qkv[:, H * dim:(H + KV) * dim].view(n, KV, dim),
         "v": qkv[:, (H + KV) * dim:].view(n, KV, dim), "pos": pos.to(torch.int32).contiguous(), "freq": freq, "sections": tuple(sections),
         "eps": 1e-6, "gain_q": None, "gain_k": None, "shift_q": None, "shift_k": None}
    if case["norm"] != "none":
        s["gain_q"], s["gain_k"] = 1 + 0.1 * rand(dim), 1 + 0.1 * rand(dim)
    if case["norm"] == "layer":
        s["shift_q"], s["shift_k"] = 0.1 * rand(dim), 0.1 * rand(dim)
    return s


def prepare(case, seed):
    g = _generator(seed)
    op, dim, kv, dtype = case["op"], case["dim"], case["kv_heads"], case["dtype"]
    if op == "rope":
        return {"case": case, **_normed_rows(case, g)}
    if op == "write":
        s = {"case": case, **_normed_rows(case, g)}
        s["slot"], pages = _slots(case["rows"], case["order"], g)
        s["read_slot"] = s["slot"].clone()
        if case["holes"]:
            s["slot"][::max(1, case["rows"] // case["holes"])] = -1
        s["pages"] = torch.zeros((pages, kv, 68 * dim), dtype=torch.uint8, device="cuda")
        return s
    if op == "read":
        slot, pages = _slots(case["rows"], case["order"], g)
        k, v = (torch.randn((pages, kv, PAGE, dim), generator=g, device="cuda").to(_TYPES[dtype]) for _ in range(2))
        return {"case": case, "slot": slot, "pages": _pages_of(k, v, dtype)}
    B, H, new, longest = case["seqs"], case["heads"], case["new"], case["longest"]
    lens = torch.randint(min(case["shortest"], longest), longest + 1, (B,), generator=g, device="cuda")
    lens[-1] = longest
    q_len = torch.full((B,), new, device="cuda")
    if case["ragged_new"]:
        q_len = 1 + torch.arange(B, device="cuda") * 7919 % new    # the same for every seed: outputs of one shape
        q_len[-1] = new
    lens = torch.maximum(q_len, lens)
    if new > 1 and B > 1:
        lens[0] = q_len[0]                                     # a sequence that begins with this chunk
    start = torch.zeros(B + 1, dtype=torch.int32, device="cuda")
    start[1:] = q_len.cumsum(0)
    per = -(-longest // PAGE)
    total = B * per
    chunk = max(1, 30_000_000 // (kv * PAGE * dim))            # pages are made some at a time: float32 temporaries stay small
    pages = torch.empty((total, kv, 68 * dim), dtype=torch.uint8, device="cuda")
    for i in range(0, total, chunk):
        n = min(chunk, total - i)
        # normed keys: a norm near sqrt(dim); values around one
        k = torch.randn((n, kv, PAGE, dim), generator=g, device="cuda").to(_TYPES[dtype])
        v = torch.randn((n, kv, PAGE, dim), generator=g, device="cuda").to(_TYPES[dtype])
        pages[i:i + n] = _pages_of(k, v, dtype)
    table = torch.randperm(total, generator=g, device="cuda").view(B, per).to(torch.int32)
    n = int(start[-1])
    q = torch.randn((n, H, dim), generator=g, device="cuda").to(_TYPES[dtype])
    return {"case": case, "q": q, "pages": pages, "table": table.contiguous(), "kv_len": lens.to(torch.int32), "q_start": start,
            "max_kv": longest, "max_q": new}


# ------------------------------------------------------------------------------------------------ plain forms

def _turned(x, gain, shift, s):
    """Norm and rotation of x [rows, heads, dim] in 64 bits, rounded to the rows' type."""
    case, dtype = s["case"], x.dtype
    x = x.double()
    if case["norm"] == "rms":
        x = x / torch.sqrt(x.square().mean(-1, keepdim=True) + s["eps"])
    elif case["norm"] == "layer":
        x = x - x.mean(-1, keepdim=True)
        x = x / torch.sqrt(x.square().mean(-1, keepdim=True) + s["eps"])
    if gain is not None:
        x = x * gain.double()
    if shift is not None:
        x = x + shift.double()
    R = case["rot"]
    axis = torch.repeat_interleave(torch.arange(len(s["sections"]), device=x.device), torch.tensor(s["sections"], device=x.device))
    angle = s["pos"].double()[:, axis] * s["freq"].double()
    c, n = torch.cos(angle).unsqueeze(1), torch.sin(angle).unsqueeze(1)
    if case["pairing"]:
        a, b = x[..., 0:R:2], x[..., 1:R:2]
        turned = torch.stack((a * c - b * n, b * c + a * n), -1).flatten(-2)
    else:
        a, b = x[..., :R // 2], x[..., R // 2:R]
        turned = torch.cat((a * c - b * n, b * c + a * n), -1)
    return torch.cat((turned, x[..., R:]), -1).to(dtype)


def _read_plain(pages, slot, dim, dtype):
    at = slot.long().clamp(min=0)
    token = torch.gather(pages[at // PAGE], 2, _token_bytes(at % PAGE, dim).unsqueeze(1).expand(-1, pages.shape[1], -1))
    kb, vb, ks, vs = token.split((dim // 2, dim // 2, dim // 32, dim // 32), -1)
    split = lambda b: torch.stack((b & 15, b >> 4), -1).flatten(-2)  # noqa: E731
    there = (slot >= 0).view(-1, 1, 1)
    k, v = _values(split(kb), ks.to(torch.int32) - 127), _values(split(vb), vs.to(torch.int32) - 127)
    return torch.where(there, k, 0.0).to(dtype), torch.where(there, v, 0.0).to(dtype)


def _write_plain(s):
    case = s["case"]
    dim = case["dim"]
    q = _turned(s["q"], s["gain_q"], s["shift_q"], s)
    k = _turned(s["k"], s["gain_k"], s["shift_k"], s)
    kc, ke = _codes(k, case["dtype"])
    vc, ve = _codes(s["v"], case["dtype"])
    token = torch.cat((kc[..., 0::2] | (kc[..., 1::2] << 4), vc[..., 0::2] | (vc[..., 1::2] << 4), (ke + 127).to(torch.uint8),
                       (ve + 127).to(torch.uint8)), -1)
    keep = s["slot"] >= 0
    at, token = s["slot"][keep].long(), token[keep]
    byte = _token_bytes(at % PAGE, dim).unsqueeze(1)
    head = torch.arange(case["kv_heads"], device=at.device).view(1, -1, 1)
    s["pages"][(at // PAGE).view(-1, 1, 1), head, byte] = token
    return q


def _attend_plain(s):
    case = s["case"]
    H, KV, dim, B = case["heads"], case["kv_heads"], case["dim"], case["seqs"]
    k, v = _sequences(s)
    new, group, L = case["new"], H // KV, k.shape[2]
    q_start = s["q_start"].long()
    q_len = q_start[1:] - q_start[:-1]
    row = torch.arange(new, device=k.device)
    valid = row < q_len.unsqueeze(1)                                                     # [B, new]
    at = (q_start[:-1].unsqueeze(1) + row).clamp(max=s["q"].shape[0] - 1)
    q = s["q"].float()[at].view(B, new, KV, group, dim).permute(0, 2, 3, 1, 4).reshape(B, KV, group * new, dim)
    score = torch.matmul(q, k.transpose(2, 3)).view(B, KV, group, new, L) * (1.0 / math.sqrt(dim))
    kv_len = s["kv_len"].long().unsqueeze(1)
    pos = kv_len - q_len.unsqueeze(1) + row                                              # [B, new]
    last = (pos if case["causal"] else (kv_len - 1).expand(-1, new)) - case["skip"]      # the last key that a row sees
    first = last - case["window"] + 1 if case["window"] else torch.zeros_like(last)
    key = torch.arange(L, device=k.device)
    seen = (key <= last.unsqueeze(-1)) & (key >= first.unsqueeze(-1)) & valid.unsqueeze(-1)
    score = score.masked_fill(~seen.view(B, 1, 1, new, L), -math.inf)
    top = score.amax(-1, keepdim=True)
    p = torch.exp(score - torch.where(top == -math.inf, 0.0, top))
    total = p.sum(-1, keepdim=True)
    o = torch.matmul(p.view(B, KV, group * new, L), v).view(B, KV, group, new, dim) / torch.where(total == 0, 1.0, total)
    o = o.permute(0, 3, 1, 2, 4).reshape(B, new, H, dim)
    return o[valid].to(s["q"].dtype)


def _sequences(s):
    """Keys and values of every sequence, [seqs, kv_heads, tokens, dim] float32."""
    case = s["case"]
    B, KV, dim = case["seqs"], case["kv_heads"], case["dim"]
    k, v = _of_pages(s["pages"][s["table"].reshape(-1).long()], dim)
    flat = lambda t: t.view(B, -1, KV, PAGE, dim).transpose(1, 2).reshape(B, KV, -1, dim)  # noqa: E731
    return flat(k), flat(v)


# ------------------------------------------------------------------------------------------------ one pass

def _opts(s, sjd):
    """The options a program keeps between its calls."""
    if "opts" not in s:
        s["opts"] = sjd.QkOpts(norm=s["case"]["norm"], eps=s["eps"], q_gain=s["gain_q"], q_shift=s["shift_q"], k_gain=s["gain_k"],
                               k_shift=s["shift_k"], rot_dim=s["case"]["rot"], adjacent=bool(s["case"]["pairing"]),
                               axis_pairs=s["sections"], freq=s["freq"])
    return s["opts"]


def run(s):
    case = s["case"]
    op, dim = case["op"], case["dim"]
    dtype = _TYPES[case["dtype"]]
    if own:
        import paper_2505_24791_amd as sjd
        if op == "rope":
            return sjd.op_qk_norm_rope(s["q"], s["k"], s["pos"], _opts(s, sjd))
        if "cache" not in s:
            s["cache"] = sjd.Kv4Cache(s["pages"], dtype)
        cache = s["cache"]
        if op == "write":
            q = sjd.op_kv4_write(cache, s["k"], s["v"], s["slot"], q=s["q"], pos=s["pos"], opts=_opts(s, sjd))
            return (q, *sjd.op_kv4_read(cache, s["read_slot"]))
        if op == "read":
            return sjd.op_kv4_read(cache, s["slot"])
        return sjd.op_kv4_attention(cache, s["q"], s["table"], s["kv_len"], q_start=s["q_start"], max_q=s["max_q"], max_kv=s["max_kv"],
                                    causal=bool(case["causal"]), skip_nearest=case["skip"], window=case["window"])
    if op == "rope":
        return _turned(s["q"], s["gain_q"], s["shift_q"], s), _turned(s["k"], s["gain_k"], s["shift_k"], s)
    if op == "write":
        return (_write_plain(s), *_read_plain(s["pages"], s["read_slot"], dim, dtype))
    if op == "read":
        return _read_plain(s["pages"], s["slot"], dim, dtype)
    return _attend_plain(s)


# ------------------------------------------------------------------------------------------------ exact results

def _turn_exact(x, gain, shift, s):
    """Norm and rotation head by head, pair by pair as complex numbers, in 64 bits."""
    case = s["case"]
    out = torch.empty(x.shape, dtype=torch.float64, device=x.device)
    unit = []
    for a, p in enumerate(s["sections"]):
        f = s["freq"][len(unit):len(unit) + p]
        unit += [torch.polar(torch.ones(x.shape[0], dtype=torch.float64, device=x.device), s["pos"][:, a].double() * w) for w in f.double()]
    for h in range(x.shape[1]):
        y = x[:, h].to(torch.float64)
        if case["norm"] != "none":
            if case["norm"] == "layer":
                y = y - y.sum(1, keepdim=True) / y.shape[1]
            y = y * (y.pow(2).sum(1, keepdim=True) / y.shape[1] + s["eps"]) ** -0.5
            y = y * gain.double()
            if shift is not None:
                y = y + shift.double()
        out[:, h] = y
    for i, u in enumerate(unit):
        a, b = (2 * i, 2 * i + 1) if case["pairing"] else (i, i + len(unit))
        z = torch.complex(out[:, :, a], out[:, :, b]) * u.unsqueeze(1)
        out[:, :, a], out[:, :, b] = z.real, z.imag
    return out


def _power64(e):
    return ((e.to(torch.int64) + 1023) << 52).view(torch.float64)


def _held_exact(x, dtype):
    """What the cache holds of x, from the definition: the nearest of the levels, the scale by trying exponents from below."""
    lo, hi = _EXPONENTS[dtype]
    g = x.double().reshape(*x.shape[:-1], -1, 32)
    top = g.abs().amax(-1)
    e = torch.full(top.shape, hi, dtype=torch.float64, device=x.device)
    for t in range(hi - 1, lo - 1, -1):
        e = torch.where(top <= 7.0 * 2.0 ** t, float(t), e)
    s = _power64(e).unsqueeze(-1)
    levels = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)
    best, off = torch.zeros_like(g), torch.full_like(g, math.inf)
    for i in (0, 2, 4, 6, 1, 3, 5, 7):                         # even levels first: they win ties
        d = (g.abs() / s - levels[i]).abs()
        best, off = torch.where(d < off, levels[i], best), torch.minimum(d, off)
    return (torch.sign(g) * best * s).reshape(x.shape)


_LEVELS = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0, -0.0, -0.5, -1.0, -1.5, -2.0, -3.0, -4.0, -6.0)


def _page_exact(pages, dim):
    """Keys and values in 64 bits, channel by channel from the table of where things are."""
    levels = torch.tensor(_LEVELS, dtype=torch.float64, device=pages.device)
    off = torch.arange(PAGE, device=pages.device)
    byte = _token_bytes(off, dim).reshape(-1)
    token = pages[..., byte].reshape(*pages.shape[:2], PAGE, -1).to(torch.int64)
    got = []
    for first, at in ((0, dim), (dim // 2, dim + dim // 32)):
        b = token[..., first:first + dim // 2]
        x = torch.empty((*b.shape[:-1], dim), dtype=torch.float64, device=pages.device)
        x[..., 0::2], x[..., 1::2] = levels[b % 16], levels[b // 16]
        e = torch.repeat_interleave(token[..., at:at + dim // 32], 32, -1)
        got.append(x * _power64(e - 127))
    return got


def _attend_exact(s):
    case = s["case"]
    H, KV, dim = case["heads"], case["kv_heads"], case["dim"]
    start, lens = s["q_start"].tolist(), s["kv_len"].tolist()
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    for b in range(case["seqs"]):
        n, L = start[b + 1] - start[b], lens[b]
        if not n or not L:
            continue
        table = s["table"][b, :-(-L // PAGE)].long()
        i = torch.arange(n, device="cuda").unsqueeze(1)
        t = torch.arange(L, device="cuda").unsqueeze(0)
        end = (L - n + i if case["causal"] else L - 1 + 0 * i) - case["skip"]
        hidden = t > end
        if case["window"]:
            hidden = hidden | (t <= end - case["window"])
        empty = hidden.all(1, keepdim=True)
        for h in range(KV):
            k, v = (x.reshape(-1, dim)[:L] for x in _page_exact(s["pages"][table, h:h + 1], dim))
            for j in range(h * (H // KV), (h + 1) * (H // KV)):
                z = s["q"][start[b]:start[b + 1], j].double() @ k.T / math.sqrt(dim)
                w = torch.softmax(z.masked_fill(hidden, -1e300), 1)
                out[start[b]:start[b + 1], j] = torch.where(empty, 0.0, w @ v)
    return out


def exact(case, seed):
    s = prepare(case, seed)
    op, dim = case["op"], case["dim"]
    if op == "rope":
        return _turn_exact(s["q"], s["gain_q"], s["shift_q"], s), _turn_exact(s["k"], s["gain_k"], s["shift_k"], s)
    if op == "write":
        dtype = _TYPES[case["dtype"]]
        there = (s["slot"] >= 0).view(-1, 1, 1)
        k = _held_exact(_turn_exact(s["k"], s["gain_k"], s["shift_k"], s).to(dtype), case["dtype"])
        v = _held_exact(s["v"], case["dtype"])
        return _turn_exact(s["q"], s["gain_q"], s["shift_q"], s), torch.where(there, k, 0.0), torch.where(there, v, 0.0)
    if op == "read":
        k, v = _page_exact(s["pages"], dim)
        at = s["slot"].long()
        return k[at // PAGE, :, at % PAGE], v[at // PAGE, :, at % PAGE]
    return _attend_exact(s)


# ------------------------------------------------------------------------------------------------ work

def work(case):
    op, dim, kv, size = case["op"], case["dim"], case["kv_heads"], 4 if case["dtype"] == "f32" else 2
    held = 17 * dim // 16                                      # bytes of a token's key and value together, for one head
    if op == "read":
        n = case["rows"] * kv
        return {"bytes": n * (held + 2 * dim * size) + 4 * case["rows"], "flops": 4 * n * dim}
    if op in ("rope", "write"):
        rows, vectors = case["rows"], case["rows"] * (case["heads"] + kv)
        moved = 4 * rows * case["axes"]
        flops = vectors * dim * (4 + 6)
        if op == "rope":
            return {"bytes": moved + 2 * vectors * dim * size, "flops": flops}
        n = rows * kv
        # queries in and out; keys and values in, held, read again and handed back
        moved += 8 * rows + 2 * rows * case["heads"] * dim * size + n * (2 * dim * size + held) + n * (held + 2 * dim * size)
        return {"bytes": moved, "flops": flops + 8 * n * dim}
    B, new, H = case["seqs"], case["new"], case["heads"]
    tokens = B * (min(case["shortest"], case["longest"]) + case["longest"]) / 2
    rows = B * (new + 1) / 2 if case["ragged_new"] else B * new
    seen = tokens / B - case["skip"] - (new / 2 if case["causal"] else 0)
    if case["window"]:
        seen = min(seen, case["window"])
        tokens = min(tokens, B * (case["window"] + new))
    return {"bytes": tokens * kv * held + 2 * rows * H * dim * size, "flops": 4 * rows * H * dim * max(1.0, seen)}

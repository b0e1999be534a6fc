"""Plain float64 forms of the head norms with rotation, of the 4-bit cache format and of attention over it (numpy, CPU)."""
import numpy as np

LEVELS = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
EXPONENTS = {"float16": (-23, 13), "bfloat16": (-125, 125), "float32": (-125, 125)}


def held(x, dtype):
    """What a cache for rows of ``dtype`` holds of x [..., dim] (float64 of values of that type)."""
    lo, hi = EXPONENTS[dtype]
    g = np.asarray(x, np.float64).reshape(*x.shape[:-1], -1, 32)
    with np.errstate(invalid="ignore"):
        top = np.abs(g).max(-1)
        bad = ~np.isfinite(g).all(-1)
        top = np.where(bad, 1.0, top)
        e = np.full(top.shape, lo)
        while True:
            more = (top > 7.0 * np.ldexp(1.0, e)) & (e < hi)
            if not more.any():
                break
            e = e + more
        s = np.ldexp(1.0, e)[..., None]
        a = np.abs(g) / s
        # nearest level, ties to the even code: between neighbours lower and upper
        up = np.searchsorted(LEVELS, np.where(np.isfinite(a), a, 0.0)).clip(1, 7)
        low = up - 1
        dl, du = a - LEVELS[low], LEVELS[up] - a
        code = np.where((dl < du) | ((dl == du) & (low % 2 == 0)), low, up)
        v = np.copysign(LEVELS[code] * s, g)
        v = np.where(bad[..., None], np.nan, v)
    return v.reshape(x.shape)


def norm_rotate(x, pos, *, norm, eps, gain, shift, rot, adjacent, axis_pairs, freq):
    """x [rows, heads, dim] float64; pos [rows, axes] ints."""
    x = np.asarray(x, np.float64).copy()
    if norm == "layer":
        x = x - x.mean(-1, keepdims=True)
    if norm in ("rms", "layer"):
        x = x / np.sqrt((x * x).mean(-1, keepdims=True) + np.float64(np.float32(eps)))
        if gain is not None:
            x = x * np.asarray(gain, np.float64)
        if shift is not None:
            x = x + np.asarray(shift, np.float64)
    y = x.copy()
    i = 0
    for axis, n in enumerate(axis_pairs if rot else ()):
        for _ in range(n):
            t = pos[:, axis].astype(np.longdouble) * np.longdouble(freq[i])        # 55 bits: exact in 64
            t = np.fmod(t, 2 * np.longdouble("3.14159265358979323846264338327950288"))
            c, s = np.cos(t).astype(np.float64)[:, None], np.sin(t).astype(np.float64)[:, None]
            a, b = (2 * i, 2 * i + 1) if adjacent else (i, i + rot // 2)
            y[..., a] = x[..., a] * c - x[..., b] * s
            y[..., b] = x[..., a] * s + x[..., b] * c
            i += 1
    return y


def attention(q, keys, values, kv_len, *, causal=True, skip=0, window=0, scale=None, visible=None):
    """q [n, heads, dim], keys and values [len, kv_heads, dim] float64, the rows being the last n of kv_len tokens.  Returns the result, sum p |v| / sum p
    and the largest sum |q k| scale, for error bounds.  visible [len]: keys on pages that exist."""
    n, H, dim = q.shape
    KV = keys.shape[1]
    scale = dim ** -0.5 if scale is None else scale
    out, mag, big = np.zeros_like(q), np.zeros_like(q), 0.0
    for i in range(n):
        last = (kv_len - n + i if causal else kv_len - 1) - skip
        first = max(0, last - window + 1) if window else 0
        t = np.arange(first, max(last, -1) + 1)
        if visible is not None:
            t = t[visible[t]]
        if not len(t):
            continue
        for h in range(H):
            k, v = keys[t, h // (H // KV)], values[t, h // (H // KV)]
            s = k @ q[i, h] * scale
            big = max(big, float(np.nanmax(np.abs(k) @ np.abs(q[i, h])) * scale)) if np.isfinite(s).any() else big
            p = np.exp(s - s.max())
            out[i, h], mag[i, h] = p @ v / p.sum(), p @ np.abs(v) / p.sum()
    return out, mag, big

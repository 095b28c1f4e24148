"""The operators of include/lba_attention.h in 64 bits with numpy, from their formulas, and how far float32 arithmetic may be from them."""
import numpy as np

U = 2.0 ** -24                       # half a unit in the last place of float32, relative
TINY = 2.0 ** -126                   # what is smaller counts as zero: a weight, a product or a sum is off by that much besides
FOURS = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def rounding(dtype):
    """A rounding to the type, relative."""
    return 2.0 ** -8 if dtype == "bf16" else U


# ---- rotary positions -----------------------------------------------------------------------

def rope(x, positions, freq, interleaved, gain, sign=1.0):
    """(y, bound) of x [T, H, D]."""
    R = 2 * len(freq)
    turn = positions.astype(np.float64)[:, None, None] * freq
    c, s = gain * np.cos(turn), gain * sign * np.sin(turn)
    y, tol = x.astype(np.float64).copy(), np.zeros(x.shape)
    i, j = (slice(0, R, 2), slice(1, R, 2)) if interleaved else (slice(0, R // 2), slice(R // 2, R))
    a, b = x[..., i].astype(np.float64), x[..., j].astype(np.float64)
    y[..., i], y[..., j] = a * c - b * s, b * c + a * s
    # the angle: its float64 product and the factor 1 / 2 pi are off by 2^-53 each, in turns of the whole angle; then a float32 rounding of an
    # angle of at most 1, the series (under 2^-28), about four roundings of its value, two of the gain, and three of the rotation
    off = abs(gain) * (4 * 2.0 ** -53 * np.abs(turn) + 12 * U) * np.ones_like(a)
    tol[..., i] = tol[..., j] = (np.abs(a) + np.abs(b)) * off
    return y, tol


# ---- attention ------------------------------------------------------------------------------

def seen(n, m, causal):
    return np.arange(m)[None] <= np.arange(n)[:, None] + (m - n) if causal else np.ones((n, m), bool)


def attend(q, k, v, see, scale, dtype, pieces=1):
    """One head of one sequence: everything the bounds need.  q [n, D], k and v [m, D], see [n, m]; hidden places of k and v must be finite.
    pieces: the parts that a float32 factor is split into, each with a product and a sum of its own."""
    q, k, v = (t.astype(np.float64) for t in (q, k, v))
    n, m, D = q.shape[0], k.shape[0], q.shape[1]
    s = scale * (q @ k.T)
    es = (pieces * D + 4) * U * abs(scale) * (np.abs(q) @ np.abs(k).T)                        # D products and sums, the scale
    z = np.where(see, s, -np.inf)
    some = see.any(1)
    top = np.where(some, z.max(1, initial=-np.inf), 0.0)
    e = np.exp(z - top[:, None])
    l = e.sum(1)
    p = e / np.where(some, l, 1.0)[:, None]
    o = p @ v
    # a weight: the score's error, roundings of the difference from a running maximum and of the exponential, which is off by 1.5 units
    dp = es + 6 * U * (np.abs(s - top[:, None]) + 1) + 8 * U
    dp = np.where(see, dp, 0.0)
    sums = (pieces * m + 8) * U                                                               # of n terms, rescaled a few times
    dl = (p * dp).sum(1) + sums
    bf = rounding(dtype) if dtype == "bf16" else 0.0
    to = (p * (dp + bf + sums)) @ np.abs(v) + np.abs(o) * (dl + 4 * U)[:, None] + 4 * TINY * (1 + np.abs(v).sum(0))
    with np.errstate(divide="ignore"):
        lse = np.where(some, top + np.log(np.where(some, l, 1.0)), -np.inf)
    tl = np.where(some, 1.1 * dl + 8 * U * (1 + np.abs(np.where(some, lse, 0.0))), 0.0)
    return {"q": q, "k": k, "v": v, "see": see, "s": s, "es": es, "p": p, "o": o, "to": 1.1 * to, "lse": lse, "tl": tl, "scale": scale, "dtype": dtype, "some": some}


def attend_bwd(f, g, tg=None):
    """(dq, dk, dv) and their bounds before the results are rounded, of one query head; tg: how far g may be off itself."""
    g = g.astype(np.float64)
    tg = np.zeros(g.shape) if tg is None else tg
    q, k, v, p, D = f["q"], f["k"], f["v"], f["p"], f["q"].shape[1]
    n, m = p.shape
    bf = 2.0 ** -8 if f["dtype"] == "bf16" else 0.0
    lse = np.where(f["some"], f["lse"], 0.0)
    dp = np.where(f["see"], f["es"] + 6 * U * (np.abs(f["s"]) + np.abs(lse)[:, None] + 1) + f["tl"][:, None], 0.0)
    u = g @ v.T
    eu = (D + 4) * U * (np.abs(g) @ np.abs(v).T) + tg @ np.abs(v).T
    delta = (g * f["o"]).sum(1)
    ed = (np.abs(g) * (f["to"] + (bf + U) * np.abs(f["o"]) * 1.01)).sum(1) + (D + 4) * U * (np.abs(g) * np.abs(f["o"])).sum(1) + (tg * np.abs(f["o"])).sum(1)
    w = u - delta[:, None]
    ds = p * w
    es = p * (dp * 1.1 * np.abs(w) + eu + ed[:, None] + 2 * U * np.abs(w)) + (bf + 2 * U) * np.abs(ds) * 1.01 + 4 * TINY * (1 + np.abs(w))
    sc = abs(f["scale"])
    dq, dk, dv = f["scale"] * (ds @ k), f["scale"] * (ds.T @ q), p.T @ g
    tq = sc * (es @ np.abs(k) + (m + 8) * U * (np.abs(ds) @ np.abs(k))) + 4 * TINY
    tk = sc * (es.T @ np.abs(q) + (n + 8) * U * (np.abs(ds).T @ np.abs(q))) + 4 * TINY
    tv = (p * (dp * 1.1 + bf + (n + 8) * U)).T @ np.abs(g) + 1.1 * p.T @ tg + 4 * TINY * (1 + np.abs(g).sum(0))
    return (dq, dk, dv), (1.1 * tq, 1.1 * tk, 1.1 * tv)


def packed(q, k, v, lens, lens_k, causal, scale, dtype, G=None, first=0, first_k=0, tG=None):
    """Everything of packed sequences: dict of (value, bound) for o, lse and, with G, dq, dk, dv.  Rows before `first` and behind the last
    sequence are zeros (-infinity in lse), with bound 0."""
    H, KV = q.shape[1], k.shape[1]
    o, to = np.zeros(q.shape), np.zeros(q.shape)
    lse, tl = np.full(q.shape[:2], -np.inf), np.zeros(q.shape[:2])
    grads = {w: (np.zeros(t.shape), np.zeros(t.shape)) for w, t in (("dq", q), ("dk", k), ("dv", v))}
    a, c = first, first_k
    for n, m in zip(lens, lens_k):
        i, j = slice(a, a + n), slice(c, c + m)
        a, c = a + n, c + m
        for h in range(H):
            kv = h // (H // KV)
            f = attend(q[i, h], k[j, kv], v[j, kv], seen(n, m, causal), scale, dtype)
            o[i, h], to[i, h], lse[i, h], tl[i, h] = f["o"], f["to"], f["lse"], f["tl"]
            if G is not None:
                for (w, r, hh), x, t in zip((("dq", i, h), ("dk", j, kv), ("dv", j, kv)), *attend_bwd(f, G[i, h], None if tG is None else tG[i, h])):
                    grads[w][0][r, hh] += x
                    grads[w][1][r, hh] += t + 2 * U * np.abs(x)                      # the sum over a group's heads
    got = {"o": (o, to), "lse": (lse, tl)}
    return {**got, **grads} if G is not None else got


# ---- the cache ------------------------------------------------------------------------------

def fours(x):
    """float32 [..., D] -> (codes uint8 [..., D / 2], scale bytes [..., D / 32])."""
    b = np.ascontiguousarray(x, np.float32).reshape(x.shape[:-1] + (-1, 32))
    a = np.abs(b.astype(np.float64))
    a = np.where(a < 2.0 ** -126, 0.0, a)
    top = a.max(-1)
    broken = ~np.isfinite(b).all(-1)
    e = np.full(top.shape, -100)
    for x2 in range(-100, 126):                          # the smallest power for which the largest element is at most 6 of it
        e = np.where((e == x2 - 1) & (top > 6 * 2.0 ** (x2 - 1)), x2, e) if x2 > -100 else e
    u = np.where(np.isfinite(a), a, 0.0) / (2.0 ** e.astype(np.float64))[..., None]
    mids = (FOURS[1:] + FOURS[:-1]) / 2
    code = np.searchsorted(mids, u)
    code += np.isin(u, mids) & (code % 2 == 1)           # the middle goes to the even code
    code = np.where(broken[..., None], 0, code + 8 * np.signbit(b)).reshape(x.shape)
    return (code[..., 0::2] + 16 * code[..., 1::2]).astype(np.uint8), np.where(broken, 255, e + 127).astype(np.uint8)


def fours_values(codes, scales):
    c = np.stack([codes & 15, codes >> 4], -1).reshape(codes.shape[:-1] + (-1,))
    v = np.where(c >= 8, -1.0, 1.0) * FOURS[c & 7]
    s = np.where(scales == 255, np.nan, np.where(scales == 0, 0.0, 2.0 ** (scales.astype(np.float64) - 127)))
    return v * np.repeat(s, 32, -1)

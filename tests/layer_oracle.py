"""The operators of include/lba_layer.h in 64 bits with numpy, element by element from their formulas, and the code formats."""
import math

import numpy as np
from scipy.special import erf as _erf

U = 2.0 ** -24                       # half a unit in the last place of float32, relative


def code_values(E, M, bias):
    c = np.arange(256)
    e, m, s = (c >> M) & ((1 << E) - 1), c & ((1 << M) - 1), np.where(c & 128, -1.0, 1.0)
    return s * np.where(e > 0, (1 + m / 2.0 ** M) * 2.0 ** (e - float(bias)), m * 2.0 ** (1 - float(bias) - M))


def nearest_code_value(v, E, M, bias):
    """The value of the format nearest to v, ties to the even code, saturated."""
    vals = code_values(E, M, bias)[:(127 if E == 4 else 128)]
    a = np.minimum(np.abs(v), vals[-1])
    hi = np.clip(np.searchsorted(vals, a), 1, len(vals) - 1)
    lo = hi - 1
    dl, dh = a - vals[lo], vals[hi] - a
    pick = np.where((dh < dl) | ((dh == dl) & (hi % 2 == 0)), hi, lo)
    return np.where(v < 0, -1.0, 1.0) * vals[pick]


def check_codes(codes, want, tol, fmt):
    """Every code stands for a value as near to the exact one as the nearest value is, but for the float32 error `tol` of what was rounded."""
    got = code_values(*fmt)[codes]
    near = nearest_code_value(want, *fmt)
    top = code_values(*fmt)[126 if fmt[0] == 4 else 127]
    w = np.clip(want, -top, top)
    bad = np.abs(got - w) > np.abs(near - w) + 2 * tol
    assert not bad.any(), (int(bad.sum()), np.argwhere(bad)[:3], got[bad][:3], want[bad][:3])


def bf16(x):
    """float64 -> nearest bfloat16 values (through float32 only where that is exact enough for test inputs)."""
    u = np.ascontiguousarray(x, dtype=np.float32).view(np.uint32).astype(np.uint64)
    u = (u + 0x7FFF + ((u >> 16) & 1)) & 0xFFFF0000
    return u.astype(np.uint32).view(np.float32)


GOLDEN = np.uint64(0x9E3779B97F4A7C15)


def _mix(z):
    z = (z ^ (z >> np.uint64(30))) * np.uint64(0xBF58476D1CE4E5B9)
    z = (z ^ (z >> np.uint64(27))) * np.uint64(0x94D049BB133111EB)
    return z ^ (z >> np.uint64(31))


def drop_base(seed, stream):
    with np.errstate(over="ignore"):
        a = _mix(np.array([(2 * seed + 1) & (2 ** 64 - 1)], dtype=np.uint64))
        return _mix(a ^ (np.array([(2 * stream + 1) & (2 ** 64 - 1)], dtype=np.uint64) * GOLDEN))


def threshold(p):
    return math.floor(65536 * p + 0.5)


def drop_factors(p, seed, stream, start, count):
    """0 or 65536 / (65536 - T) for elements start .. start + count - 1."""
    T = threshold(p)
    first = start // 4
    with np.errstate(over="ignore"):
        w = _mix(np.arange(first, (start + count + 3) // 4 + 1, dtype=np.uint64) * GOLDEN + drop_base(seed, stream))
    u = w.view(np.uint16)[start - 4 * first:][:count]
    return np.where(u >= T, 65536.0 / max(1, 65536 - T), 0.0)


def act(z, kind):
    """(value, slope); kind: 0 none, 1 relu, 2 gelu, 3 silu."""
    if kind == 1:
        return np.maximum(z, 0.0), (z > 0).astype(np.float64)
    if kind == 2:
        phi = 0.5 * (1 + _erf(z / math.sqrt(2.0)))
        return z * phi, phi + z * np.exp(-0.5 * z * z) / math.sqrt(2 * math.pi)
    if kind == 3:
        h = 1 / (1 + np.exp(-z))
        return z * h, h * (1 + z * (1 - h))
    return z, np.ones_like(z)


def norm(x, gamma, beta, eps):
    """(y, mean, rstd, tol): tol bounds the float32 error of a sum of N terms in chains of at most 32 + N / 1024."""
    n = x.shape[-1]
    mean = x.mean(-1, keepdims=True)
    rstd = 1 / np.sqrt(((x - mean) ** 2).mean(-1, keepdims=True) + eps)
    g = np.ones(n) if gamma is None else gamma
    b = np.zeros(n) if beta is None else beta
    y = (x - mean) * rstd * g + b
    depth = 64 + n / 512
    tol = depth * U * (np.abs(g) * rstd * (np.abs(x).mean(-1, keepdims=True) + np.abs(x)) + np.abs((x - mean) * rstd * g) + np.abs(b)) + 1e-37
    return y, mean[..., 0], rstd[..., 0], tol


def norm_bwd(G, x, gamma, mean, rstd):
    """(dx, dgamma, dbeta) and their bounds, from the mean and rstd that the forward call stored."""
    m, n = x.shape
    g = np.ones(n) if gamma is None else gamma
    u = (x - mean[:, None]) * rstd[:, None]
    h = G * g
    mh, mhu = h.mean(-1, keepdims=True), (h * u).mean(-1, keepdims=True)
    dx = rstd[:, None] * (h - mh - u * mhu)
    depth = 64 + n / 512
    tx = depth * U * rstd[:, None] * (np.abs(h) + np.abs(h).mean(-1, keepdims=True) + np.abs(u) * np.abs(h * u).mean(-1, keepdims=True)) + 1e-37
    return (dx, (G * u).sum(0), G.sum(0)), (tx, (m + 64) * U * np.abs(G * u).sum(0) + 1e-37, (m + 64) * U * np.abs(G).sum(0) + 1e-37)


def dense(A, B, fa, fb, bias, act_kind, gated, f, residual):
    """(y, tol, parts): the product of codes and what follows it; f: the dropout factors or None.  A sum of K exact products in float32 is off
    by at most (K + 16) U of the sum of their magnitudes; activations change by at most 1.2 of what their argument does."""
    a, b = code_values(*fa)[A], code_values(*fb)[B]
    K = a.shape[1]
    z, za = a @ b.T, np.abs(a) @ np.abs(b).T
    tz = (K + 16) * U * za
    if bias is not None:
        z, tz = z + bias, tz + 2 * U * (np.abs(z) + np.abs(bias))
    n = z.shape[1] // 2 if gated else z.shape[1]
    v, slope = act(z[:, :n], act_kind)
    tv = 1.2 * tz[:, :n] + 16 * U * (np.abs(z[:, :n]) + np.abs(v))
    y, ty = v, tv
    if gated:
        u, tu = z[:, n:], tz[:, n:]
        y, ty = v * u, tv * np.abs(u) + (np.abs(v) + tv) * tu + 2 * U * np.abs(v * u)
    if f is not None:
        y, ty = y * f, (ty + 2 * U * np.abs(y)) * f
    if residual is not None:
        y, ty = y + residual, ty + 2 * U * (np.abs(y) + np.abs(residual))
    return y, ty + 1e-37, dict(a=a, b=b, z=z, tz=tz, v=v, tv=tv, slope=slope, n=n, f=f, gated=gated, act=act_kind)


def dense_bwd(G, parts, rounded):
    """((dA, dB, dbias), their bounds).  `rounded`: the gradient of the sums is rounded to bfloat16 before the products."""
    a, b, z, n = parts["a"], parts["b"], parts["z"], parts["n"]
    g = G if parts["f"] is None else G * parts["f"]
    ts = 1.2 * parts["tz"][:, :n] + 24 * U
    if parts["act"] == 1:                                   # a sum within its error of the corner may fall on either side
        ts = np.where(np.abs(z[:, :n]) <= parts["tz"][:, :n], 1.0, 0.0) + 2 * U
    if parts["act"] == 0:
        ts = 2 * U * np.ones_like(ts)
    if parts["gated"]:
        u, tu = z[:, n:], parts["tz"][:, n:]
        d = np.concatenate([g * u * parts["slope"], g * parts["v"]], 1)
        t = np.concatenate([np.abs(g) * (ts * (np.abs(u) + tu) + np.abs(parts["slope"]) * tu), np.abs(g) * parts["tv"]], 1) + 4 * U * np.abs(d)
    else:
        d = g * parts["slope"]
        t = np.abs(g) * ts + 4 * U * np.abs(d)
    m, cols = d.shape
    db, tb = d.sum(0), t.sum(0) + (m + 64) * U * np.abs(d).sum(0)
    t = t + (2.0 ** -8 if rounded else 0.0) * np.abs(d)
    dA, dB = d @ b, d.T @ a
    tA = t @ np.abs(b) + (3 * cols + 16) * U * (np.abs(d) @ np.abs(b))
    tB = t.T @ np.abs(a) + (3 * m + 16) * U * (np.abs(d).T @ np.abs(a))
    return (dA, dB, db), (tA + 1e-37, tB + 1e-37, tb + 1e-37)

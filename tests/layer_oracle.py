"""The operators of include/lba_layer.h in 64 bits with numpy, element by element from their formulas, and the code formats."""
import math

import numpy as np

U = 2.0 ** -24                       # half a unit in the last place of float32, relative
_erf = np.vectorize(math.erf, otypes=[np.float64])


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

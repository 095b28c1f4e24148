"""Gradients of attention in bfloat16 where G . V^T - rowsum(G * O) cancels: few keys, and values with a mean, whose rounded outputs say too little about that sum."""
import numpy as np
import pytest
import torch

import attention_oracle as ao
from attention_oracle import TINY, U
from paper_2401_14110_amd import binding as lb
from test_gpu_attention import starts
from test_gpu_layernorm import dev, host, values

BF, TILE, FEW = 2.0 ** -8, 128, 512  # a rounding to bfloat16; queries of a tile; keys up to which their sum is made again


def gradients(f, g, few):
    """(dq, dk, dv) and their bounds of one query head, as ao.attend_bwd has them; for the queries `few` the sum of P * (G . V^T) is one in float32 (an error
    of each term, its products' and its sum's), for the others one over an O that is rounded."""
    g = g.astype(np.float64)
    q, k, v, p, D = f["q"], f["k"], f["v"], f["p"], f["q"].shape[1]
    n, m = p.shape
    lse = np.where(f["some"], f["lse"], 0.0)
    dp = np.where(f["see"], f["es"] + 6 * U * (np.abs(f["s"]) + np.abs(lse)[:, None] + 1) + f["tl"][:, None], 0.0)
    u = g @ v.T
    eu = (D + 4) * U * (np.abs(g) @ np.abs(v).T)
    delta = (p * u).sum(1)
    own = (p * (1.1 * dp * np.abs(u) + eu + (m + 8) * U * np.abs(u))).sum(1) + 4 * TINY * (1 + np.abs(u).sum(1))
    other = (np.abs(g) * (f["to"] + (BF + U) * np.abs(f["o"]) * 1.01)).sum(1) + (D + 4) * U * (np.abs(g) * np.abs(f["o"])).sum(1)
    ed = np.where(few, own, other)
    w = u - delta[:, None]
    ds = p * w
    es = p * (dp * 1.1 * np.abs(w) + eu + ed[:, None] + 2 * U * np.abs(w)) + (BF + 2 * U) * np.abs(ds) * 1.01 + 4 * TINY * (1 + np.abs(w))
    sc = abs(f["scale"])
    tq = sc * (es @ np.abs(k) + (m + 8) * U * (np.abs(ds) @ np.abs(k))) + 4 * TINY
    tk = sc * (es.T @ np.abs(q) + (n + 8) * U * (np.abs(ds).T @ np.abs(q))) + 4 * TINY
    tv = (p * (dp * 1.1 + BF + (n + 8) * U)).T @ np.abs(g) + 4 * TINY * (1 + np.abs(g).sum(0))
    return (f["scale"] * (ds @ k), f["scale"] * (ds.T @ q), p.T @ g), (1.1 * tq, 1.1 * tk, 1.1 * tv)


@pytest.mark.gpu
@pytest.mark.parametrize("mean", [0.0, 8.0, 64.0])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("lens,lens_k,H,KV,D", [
    ([2, 1, 3], [2, 1, 3], 2, 1, 64), ([64, 65, 128], [64, 65, 128], 2, 2, 64), ([5, 130], [70, 129], 4, 2, 83), ([200, 33], [200, 33], 2, 1, 128), ([300], [512], 1, 1, 96),
    ([70], [449], 2, 2, 32), ([3, 0, 9], [0, 5, 513], 2, 1, 40), ([90, 1], [30, 1], 2, 2, 80),
    # cut into parts, with short sequences and early tiles among them
    ([1500, 100], [1500, 100], 2, 1, 64), ([40, 700, 1], [300, 900, 3000], 1, 1, 128)])
def test_gradients_of_values_with_a_mean(lens, lens_k, H, KV, D, causal, mean):
    against_the_formulas(lens, lens_k, H, KV, D, causal, mean, False)


def against_the_formulas(lens, lens_k, H, KV, D, causal, mean, fine):
    rng = np.random.default_rng(sum(lens) + D)
    T, Tk = sum(lens), sum(lens_k)
    q, k, G = (values(rng, (t, h, D), "bf16") for t, h in ((T, H), (Tk, KV), (T, H)))
    v = torch.from_numpy(values(rng, (Tk, KV, D), "bf16") + np.float32(mean)).bfloat16().float().numpy()
    kw = dict(starts=starts(lens), starts_k=starts(lens_k), causal=causal)
    tensors = [dev(x, "bf16") for x in (q, k, v)]
    o, lse = lb.attention(*tensors, want_stats=True, **kw)
    got = [host(t) for t in lb.attention_bwd(dev(G, "bf16"), *tensors, o, lse, fine=fine, **kw)]
    want, tol = ([np.zeros(t.shape) for t in (q, k, v)] for _ in range(2))
    a = c = 0
    for n, m in zip(lens, lens_k):
        i, j = slice(a, a + n), slice(c, c + m)
        a, c = a + n, c + m
        see = ao.seen(n, m, causal)
        last = np.minimum(np.arange(n) // TILE * TILE + TILE, n) - 1                 # of a query's tile: it sees most
        few = (see.sum(1)[last] <= FEW) | fine if n else np.zeros(0, bool)
        for h in range(H):
            kv = h // (H // KV)
            f = ao.attend(q[i, h], k[j, kv], v[j, kv], see, float(np.float32(D ** -0.5)), "bf16")
            for at, x, t in zip((0, 1, 2), *gradients(f, G[i, h], few)):
                r, hh = (i, h) if at == 0 else (j, kv)
                want[at][r, hh] += x
                tol[at][r, hh] += t + 2 * U * np.abs(x)
    for x, w, t, name in zip(got, want, tol, ("dq", "dk", "dv")):
        assert (np.abs(x - w) <= t + BF * np.abs(w)).all(), (name, float((np.abs(x - w) / (t + BF * np.abs(w) + TINY)).max()))

"""Infinities and NaN in keys, values, queries and their gradients that some rows see and others do not: who does not see them has the bits that zeros in their place
give, who does has what the sums make of them, in the columns that hold them; and however many there are, a call takes no longer than a few times its own."""
import time

import numpy as np
import pytest
import torch

from paper_2401_14110_amd import binding as lb

DT = [torch.float32, torch.bfloat16]
INF, NAN = float("inf"), float("nan")


def ints(*v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def inputs(lens, H, KV, D, dtype, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    s = ints(*np.cumsum([0] + lens))
    return s, [torch.randn(sum(lens), h, D, device="cuda", generator=g).to(dtype) for h in (H, KV, KV, H)]


LENS = [[150], [64, 33, 129], [700], [31, 0, 1, 260], [1500]]        # (one, some and many steps, whole and cut into parts)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", DT)
@pytest.mark.parametrize("D", [16, 64, 83, 96, 128])
@pytest.mark.parametrize("lens", LENS)
def test_values(lens, D, dtype):
    H, KV = 2, 1
    s, (q, k, v, _) = inputs(lens, H, KV, D, dtype)
    clean = lb.attention(q, k, v, starts=s, want_stats=True)
    rng = np.random.default_rng(sum(lens) + D)
    T = sum(lens)
    bad = v.clone()
    spots = [(int(t), int(d), float(rng.choice([INF, -INF, NAN]))) for t, d in zip(rng.integers(0, T, 12), rng.integers(0, D, 12))]
    spots += [(T - 1, 0, NAN), (max(0, T - 2), 1, INF), (T - 1, 1, -INF), (T // 2, D - 1, -INF)]
    for t, d, x in spots:
        bad[t, 0, d] = x
    zero = torch.where(bad.isfinite(), bad, 0.0)
    want, stats = lb.attention(q, k, zero, starts=s, want_stats=True)
    got, lse = lb.attention(q, k, bad, starts=s, want_stats=True)
    assert torch.equal(lse, stats) and torch.equal(stats, clean[1])
    # per element: the sum of the infinities that its query sees; weights are positive here
    seen, at = torch.zeros(want.shape, device="cuda"), 0
    for n in lens:
        seen[at:at + n] = torch.cumsum(torch.where(bad[at:at + n].isfinite(), 0.0, bad[at:at + n].float()), 0)
        at += n
    for out in (got, lb.attention(q, k, bad, starts=s, out_dtype=torch.float32), lb.attention(q, k, bad, starts=s, fine=True)):
        assert torch.equal(out.isnan(), seen.isnan()) and torch.equal(out == INF, seen == INF) and torch.equal(out == -INF, seen == -INF)
    fine = seen == 0
    assert bool(fine.any()) and torch.equal(got[fine], want[fine])


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", DT)
@pytest.mark.parametrize("lens", LENS)
@pytest.mark.parametrize("x", [INF, NAN])
def test_keys_queries_and_gradients(lens, x, dtype):
    """What a broken row does not reach is what it is with that row zero, bit for bit."""
    s, (q, k, v, G) = inputs(lens, 4, 2, 64, dtype, 1)
    o, lse = lb.attention(q, k, v, starts=s, want_stats=True)
    base = lb.attention_bwd(G, q, k, v, o, lse, starts=s)
    first = 0
    for n in lens:
        for where in sorted({0, n // 3, n // 2, n - 1} if n > 1 else {0} if n else ()):
            t, end = first + where, first + n
            # a key and its value: queries before it, and the other sequences
            bk, bv = k.clone(), v.clone()
            bk[t, 0, ::3], bv[t, 0, 1::2] = x, -x
            ck, cv = k.clone(), v.clone()
            ck[t, 0, ::3], cv[t, 0, 1::2] = 0.0, 0.0
            got, st = lb.attention(q, bk, bv, starts=s, want_stats=True)
            want, sw = lb.attention(q, ck, cv, starts=s, want_stats=True)
            free = torch.ones(len(q), dtype=torch.bool, device="cuda")
            free[t:end] = False
            assert torch.equal(got[free], want[free]) and torch.equal(st[free], sw[free]) and torch.equal(got[:, 2:], want[:, 2:])
            assert not got[t:end, :2].isfinite().all(-1).any()
            dq = lb.attention_bwd(G, q, bk, bv, got, st, starts=s)[0]
            assert torch.equal(dq[free], lb.attention_bwd(G, q, ck, cv, want, sw, starts=s)[0][free])
            # a query and its output's gradient: keys behind it, and the other sequences
            bq, bg = q.clone(), G.clone()
            bq[t, 1, 2::5], bg[t, 1, ::2] = x, -x
            cg = G.clone()
            cg[t, 1] = 0.0
            ob, lb_ = lb.attention(bq, k, v, starts=s, want_stats=True)
            _, dk, dv = lb.attention_bwd(bg, bq, k, v, ob, lb_, starts=s)
            _, wk, wv = lb.attention_bwd(cg, q, k, v, o, lse, starts=s)
            free = torch.ones(len(q), dtype=torch.bool, device="cuda")
            free[first:t + 1] = False
            assert torch.equal(dk[free], wk[free]) and torch.equal(dv[free], wv[free]) and torch.equal(dk[:, 1], base[1][:, 1]) and torch.equal(dv[:, 1], base[2][:, 1])
            assert not dv[first:t + 1, 0].isfinite().all(-1).any()
            if n > 1 and where:                          # (a query that sees one key leaves nothing to dK)
                assert not dk[first:t + 1, 0].isfinite().all(-1).any()
        first += n


@pytest.mark.gpu
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("dtype", DT)
@pytest.mark.parametrize("fine", [False, True])
def test_columns_of_infinities(fine, dtype, causal):
    """Whole columns, under weights of up to 2^8: none of their pieces makes a NaN of them."""
    n, D = 300, 64
    g = torch.Generator(device="cuda").manual_seed(3)
    q = torch.rand(n, 1, D, device="cuda", generator=g).add_(0.5).to(dtype)
    k = (torch.rand(n, 1, D, device="cuda", generator=g) + torch.linspace(0, 3, n, device="cuda")[:, None, None]).to(dtype)          # the maximum rises with the keys
    v = torch.randn(n, 1, D, device="cuda", generator=g).to(dtype)
    v[:, 0, 3], v[:, 0, 4], v[::7, 0, 5] = INF, -INF, -INF
    for out in (dtype, torch.float32):
        o = lb.attention(q, k, v, causal=causal, fine=fine, out_dtype=out)
        assert (o[..., 3] == INF).all() and (o[..., 4] == -INF).all() and (o[..., 5] == -INF).all() and o[..., :3].isfinite().all() and o[..., 6:].isfinite().all()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", DT)
def test_nothing_but_nan(dtype):
    """A step that has diverged: each tile row by row over all that it sees would take minutes here."""
    n, H, KV, D = 16384, 8, 2, 64
    s, (q, k, v, G) = inputs([n], H, KV, D, dtype)
    for t in (q, k, v, G):
        t[:, :, ::2] = NAN

    def step():
        torch.cuda.synchronize()
        begin = time.monotonic()
        o, lse = lb.attention(q, k, v, starts=s, want_stats=True)
        d = lb.attention_bwd(G, q, k, v, o, lse, starts=s)
        torch.cuda.synchronize()
        return time.monotonic() - begin, (o, lse) + tuple(d)

    _, outs = step()
    assert all(t.isnan().all() for t in outs[:2] + outs[2:3])
    broken, _ = step()
    for t in (q, k, v, G):
        t.nan_to_num_(0.0)
    step()
    clean, _ = step()
    assert broken < 20 * clean + 0.1

"""The feed-forward block on codes: its outputs and gradients against the formulas in 64 bits at the codes that it used, with every
bound from the number of float32 sums and roundings that an output goes through."""
import numpy as np
import pytest
import torch

import layer_oracle as lo
from oracle import lba_grad_ref, lba_ref
from paper_2401_14110_amd import binding as lb
from paper_2401_14110_amd import feed_forward as ff
from paper_2401_14110_amd import inputs

pytestmark = pytest.mark.gpu


def host(t):
    return t.detach().cpu().numpy().astype(np.float64)


def near(got, want, tol, what):
    err = np.abs(host(got) - want)
    assert (err <= tol).all(), (what, float((err / tol).max()))


def check_first(block, x, kept):
    """The codes n and u that the forward call kept, against norm and product in 64 bits; returns u's parts."""
    q = {k: host(v) for k, v in block.params.items()}
    n, u, mean, rstd = kept[1].cpu().numpy(), kept[2].cpu().numpy(), host(kept[3]), host(kept[4])
    f_n, f_u, f_1 = (ff.scaled_format(t) for t in (block.t_n, block.t_u, block.t_1))
    y, m, r, tol = lo.norm(host(x), q["gamma"], q["beta"], block.eps)
    lo.check_codes(n, y, tol, f_n)
    assert np.abs(mean - m).max() <= 1e-6 and np.abs(rstd / r - 1).max() <= 1e-5
    v, tol, parts = lo.dense(n, block.w1.cpu().numpy(), f_n, f_1, q["b1"], block.act, block.gated, None, None)
    lo.check_codes(u, v, tol, f_u)
    return q, parts, mean, rstd


def check_grads(block, x, kept, G, du, tdu, dx, grads, q, parts, mean, rstd):
    """What follows the second product's gradient du (float32, off by tdu at most)."""
    (dn, dw1, db1), (tn, tw, tb) = lo.dense_bwd(du, parts, False)
    n = parts["n"]
    spread = np.abs(parts["slope"]) * 1.01 + 1e-6        # what an error of du does to the gradient of the sums
    e = [tdu * spread * np.abs(parts["z"][:, n:]), tdu * np.abs(parts["v"])] if parts["gated"] else [tdu * spread]
    e = np.concatenate(e, 1)
    tn, tw, tb = tn + e @ np.abs(parts["b"]), tw + e.T @ np.abs(parts["a"]), tb + e.sum(0)
    near(grads["w1"], dw1, tw, "w1")
    near(grads["b1"], db1, tb, "b1")
    (dxn, dg, db), (tx, tg, tbeta) = lo.norm_bwd(dn, host(x), q["gamma"], mean, rstd)
    u = (host(x) - mean[:, None]) * rstd[:, None]
    h = tn * np.abs(q["gamma"])
    tx = tx + rstd[:, None] * (h + h.mean(1, keepdims=True) + np.abs(u) * (h * np.abs(u)).mean(1, keepdims=True)) + 2 * lo.U * np.abs(dxn + G)
    near(dx, dxn + G, tx, "dx")
    near(grads["gamma"], dg, tg + (tn * np.abs(u)).sum(0), "gamma")
    near(grads["beta"], db, tbeta + tn.sum(0), "beta")


@pytest.mark.parametrize("rows,width,hidden,act,gated,p", [
    (33, 40, 72, lb.ACT_GELU, False, 0.1), (130, 257, 131, lb.ACT_SILU, True, 0.25), (70, 64, 256, lb.ACT_NONE, False, 0.0)])
def test_training_step(rows, width, hidden, act, gated, p):
    block = ff.FeedForward(width, hidden, act=act, gated=gated, p=p, seed=rows)
    rng = np.random.default_rng(rows)
    x = torch.from_numpy(rng.standard_normal((rows, width)).astype(np.float32)).cuda()
    G = rng.standard_normal((rows, width)).astype(np.float32)
    y, kept = block.forward(x, seed=5, train=True)
    q, parts, mean, rstd = check_first(block, x, kept)
    f_u, f_2 = ff.scaled_format(block.t_u), ff.scaled_format(block.t_2)
    f = lo.drop_factors(p, 5, 0, 0, rows * width).reshape(rows, width) if p else None
    want, tol, second = lo.dense(kept[2].cpu().numpy(), block.w2.cpu().numpy(), f_u, f_2, q["b2"], 0, False, f, host(x))
    near(y, want, tol, "y")
    dx, grads = block.backward(torch.from_numpy(G).cuda(), kept)
    (du, dw2, db2), (tu, tw, tb) = lo.dense_bwd(G.astype(np.float64), second, False)
    near(grads["w2"], dw2, tw, "w2")
    near(grads["b2"], db2, tb, "b2")
    check_grads(block, x, kept, G.astype(np.float64), du, tu, dx, grads, q, parts, mean, rstd)


def test_simulated_accumulators():
    rows, width, hidden, p = 37, 48, 96, 0.1
    block = ff.FeedForward(width, hidden, p=p, accumulator=((5, 7, 15), (4, 7, 16)), seed=3)       # sums beyond 1 overflow
    rng = np.random.default_rng(3)
    x = torch.from_numpy(rng.standard_normal((rows, width)).astype(np.float32)).cuda()
    G = rng.standard_normal((rows, width)).astype(np.float32)
    y, kept = block.forward(x, seed=9, train=True)
    q, parts, mean, rstd = check_first(block, x, kept)
    u, w2 = kept[2].cpu().numpy(), block.w2.cpu().numpy()
    qprod, qacc, t = inputs.folded_formats(block.t_u, block.t_2, *block.accumulator)
    fp, fa = lba_ref.QFmt(*qprod), lba_ref.QFmt(*qacc)
    c, of, _ = lba_ref.gemm_bwd(u, w2, fp, fa)
    assert of.any()
    f = lo.drop_factors(p, 9, 0, 0, rows * width).reshape(rows, width)
    z = c.astype(np.float64) * 2.0 ** -t + q["b2"]
    want = z * f + host(x)
    near(y, want, 4 * lo.U * (np.abs(z) * f + np.abs(host(x)) + np.abs(q["b2"]) * f) + 1e-37, "y")
    dx, grads = block.backward(torch.from_numpy(G).cuda(), kept)
    dz = (G.astype(np.float64) * f).astype(np.float32)
    gx, gw = lba_grad_ref.grad(dz, u, w2, fp, fa, 1)
    ax, aw = lba_grad_ref.grad_abs(dz, u, w2, fp, fa, 1)
    # sums in float32 of dz's own rounding, which is 2 U at most
    tx, tw = (2 * (width + 1) + 4) * lo.U * ax * 2.0 ** -block.t_2 + 1e-30, (2 * (rows + 1) + 4) * lo.U * aw * 2.0 ** -block.t_u + 1e-30
    near(grads["w2"], gw * 2.0 ** -block.t_u, tw, "w2")
    near(grads["b2"], dz.astype(np.float64).sum(0), (rows + 64) * lo.U * np.abs(dz).sum(0) + 1e-37, "b2")
    check_grads(block, x, kept, G.astype(np.float64), gx * 2.0 ** -block.t_2, tx, dx, grads, q, parts, mean, rstd)


def test_tokens_give_what_the_batch_gives():
    """One token at a time, without dropout: rows do not depend on how many go together, but for the order of float32 sums."""
    block = ff.FeedForward(96, 160, gated=True, act=lb.ACT_SILU, p=0.3, seed=1)
    x = torch.randn((80, 96), generator=torch.Generator().manual_seed(2)).cuda()
    whole = block.forward(x)
    q = {k: host(v) for k, v in block.params.items()}
    f_u, f_2 = ff.scaled_format(block.t_u), ff.scaled_format(block.t_2)
    for i in (0, 41, 79):
        y, kept = block.forward(x[i:i + 1], train=True)  # (with dropout: for the codes)
        want, tol, _ = lo.dense(kept[2].cpu().numpy(), block.w2.cpu().numpy(), f_u, f_2, q["b2"], 0, False, None, host(x[i:i + 1]))
        one = block.forward(x[i:i + 1])
        near(one, want, tol, "token")
        # where a code of u fell on the other side of a tie, the outputs differ by that step
        assert np.abs(host(one) - host(whole[i:i + 1])).max() <= 0.05 * np.abs(want).max()


@pytest.mark.parametrize("args", [[], ["--gated"], ["--simulated"]])
def test_example_learns(args):
    losses = ff.main(["--steps", "12", "--rows", "256", "--width", "64"] + args)
    assert losses[-1] < 0.9 * losses[0]

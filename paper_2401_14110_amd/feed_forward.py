"""A feed-forward block of a transformer layer on 8-bit codes, from the operators of include/lba_layer.h and the simulated product.

    y = x + dropout(u W2^T + b2),   u = act(n W1^T + b1)  or, gated,  act(n Wg^T + bg) * (n Wu^T + bu),   n = layernorm(x)

n, u and the weights are codes; each operator writes the codes that the next one reads.  The last product is the dense one, or the
simulated one where an accumulator is given; its gradient is then the immediate estimator's.  What rounding to codes does is passed
straight through in the backward pass.  The same calls serve one token and train on thousands.

    python -m paper_2401_14110_amd.feed_forward [--steps 20] [--rows 512] [--width 256] [--gated] [--simulated]
"""
import argparse
import math

import torch

from . import binding as lba
from . import inputs

_E4M3_TOP = 448.0


def scaled_format(t):
    """E4M3 codes of x * 2^t."""
    return (4, 3, 7 + t)


def scale_of(w):
    """The largest t for which w * 2^t stays within the E4M3 codes (reads w back: once, where the scale is chosen)."""
    top = float(w.abs().max())
    return math.floor(math.log2(_E4M3_TOP / top)) if top > 0 else 0


def codes_of(w, t):
    return lba.dropout(w, None, out_dtype=torch.uint8, out_fmt=scaled_format(t))


class FeedForward:
    """Parameters are float32 tensors (`params`), `refresh` makes the weights' codes from them.  `accumulator` = (prod, acc) formats
    (E, M, bias) in real units makes the second product a simulated one."""

    def __init__(self, width, hidden, act=lba.ACT_GELU, gated=False, p=0.1, eps=1e-5, accumulator=None, seed=0, device="cuda"):
        g = torch.Generator().manual_seed(seed)
        rows = 2 * hidden if gated else hidden
        self.act, self.gated, self.p, self.eps, self.accumulator = act, gated, p, eps, accumulator
        p = {"gamma": torch.ones(width), "beta": torch.zeros(width),
             "w1": torch.randn((rows, width), generator=g) / math.sqrt(width), "b1": torch.zeros(rows),
             "w2": torch.randn((width, hidden), generator=g) / math.sqrt(hidden), "b2": torch.zeros(width)}
        self.params = {k: v.to(device) for k, v in p.items()}
        self.t_n, self.t_u = 5, 4                        # normalised rows and activations: up to 14 and 28 in size
        self.t_1, self.t_2 = scale_of(p["w1"]) - 1, scale_of(p["w2"]) - 1            # room for the weights to double
        self.refresh()

    def refresh(self):
        self.w1, self.w2 = codes_of(self.params["w1"], self.t_1), codes_of(self.params["w2"], self.t_2)

    def drop(self, seed, train):
        return (self.p, seed, 0) if train and self.p > 0 else None

    def forward(self, x, seed=0, train=False):
        """y of x [..., width], and with train what `backward` reads."""
        q = self.params
        f_n, f_u, f_1, f_2 = (scaled_format(t) for t in (self.t_n, self.t_u, self.t_1, self.t_2))
        drop = self.drop(seed, train)
        n = lba.layernorm(x, q["gamma"], q["beta"], self.eps, out_dtype=torch.uint8, out_fmt=f_n, want_stats=train)
        n, mean, rstd = n if train else (n, None, None)
        u = lba.dense(n, self.w1, f_n, f_1, bias=q["b1"], act=self.act, gated=self.gated, out_dtype=torch.uint8, out_fmt=f_u)
        of = None
        if self.accumulator is None:
            y = lba.dense(u, self.w2, f_u, f_2, bias=q["b2"], drop=drop, residual=x, out_dtype=x.dtype)
        else:
            qprod, qacc, t = inputs.folded_formats(self.t_u, self.t_2, *self.accumulator)
            u2 = u.view(-1, u.shape[-1])
            if train:
                c, of, _ = lba.gemm_bwd(u2, self.w2, qprod, qacc, want_uf=False)
            else:
                c = lba.gemm(u2, self.w2, qprod, qacc)
            y = lba.dropout(c.view(x.shape), drop, bias=q["b2"], residual=x, scale=2.0 ** -t, out_dtype=x.dtype)
        return (y, (x, n, u, mean, rstd, drop, of)) if train else y

    def backward(self, G, kept):
        """(dx, the gradients of `params`) for dL/dy = G and what `forward` kept."""
        q, (x, n, u, mean, rstd, drop, of) = self.params, kept
        f_n, f_u, f_1, f_2 = (scaled_format(t) for t in (self.t_n, self.t_u, self.t_1, self.t_2))
        d = {}
        if of is None:
            du, d["w2"], d["b2"] = lba.dense_bwd(G, u, self.w2, f_u, f_2, drop=drop, want_dbias=True)
        else:
            dz, d["b2"] = lba.dropout_bwd(G, drop, out_dtype=torch.float32, want_dbias=True)
            du, dw = lba.grad(dz.view(-1, dz.shape[-1]), u.view(-1, u.shape[-1]), self.w2, lba.STE_IMMEDIATE_OF, of_plane=of)
            du, d["w2"] = du.mul_(2.0 ** -self.t_2).view(u.shape), dw.mul_(2.0 ** -self.t_u)
        dn, d["w1"], d["b1"] = lba.dense_bwd(du, n, self.w1, f_n, f_1, bias=q["b1"], act=self.act, gated=self.gated, want_dbias=True)
        dx, d["gamma"], d["beta"] = lba.layernorm_bwd(dn, x, q["gamma"], mean, rstd)
        return dx.add_(G), d

    def step(self, grads, rate):
        for k, w in self.params.items():
            w.add_(grads[k], alpha=-rate)
        self.refresh()


def main(argv=None):
    ap = argparse.ArgumentParser(description="trains a feed-forward block on a fixed map and runs one token through it")
    ap.add_argument("--steps", type=int, default=20)
    ap.add_argument("--rows", type=int, default=512)
    ap.add_argument("--width", type=int, default=256)
    ap.add_argument("--rate", type=float, default=None, help="learning rate (1 / width)")
    ap.add_argument("--gated", action="store_true")
    ap.add_argument("--simulated", action="store_true", help="12-bit accumulators in the second product")
    a = ap.parse_args(argv)
    block = FeedForward(a.width, 4 * a.width, act=lba.ACT_SILU if a.gated else lba.ACT_GELU, gated=a.gated, p=0.05,
                        accumulator=((5, 7, 15), (4, 7, 7)) if a.simulated else None)
    g = torch.Generator().manual_seed(1)
    x = torch.randn((a.rows, a.width), generator=g).cuda()
    target = (x.cpu() @ (torch.randn((a.width, a.width), generator=g) / math.sqrt(a.width))).cuda()
    losses = []
    for i in range(a.steps):
        y, kept = block.forward(x, seed=i, train=True)
        err = y - target
        losses.append((err * err).mean())
        _, grads = block.backward(err * (2.0 / a.rows), kept)
        block.step(grads, a.rate or 1.0 / a.width)
    losses = [float(v) for v in losses]
    token = block.forward(x[:1])
    print("loss %.4f -> %.4f; one token: error %.4f" % (losses[0], losses[-1], float(((token - target[:1]) ** 2).mean())))
    return losses


if __name__ == "__main__":
    main()

"""What the operators around the products of a transformer layer are timed on: calls of paper_2401_14110_amd.binding on device
tensors as a user's program makes them, and the same operators in plain torch operations.

  layernorm   y = (x - mean) / sqrt(var + eps) * gamma + beta over the last axis, and its gradients
  dropout     y = residual + keep * act(scale * x + bias) / (1 - p), the mask made from (seed, stream, index) and never stored,
              and its gradients
  dense       y = residual + keep * act(A . B^T + bias) / (1 - p) on 8-bit codes with wide accumulators, and its gradients
  gated       the same with act(A . Bg^T + bg) * (A . Bu^T + bu), B and bias holding the gate's rows first

`own` says which of the two run() computes; it is set from outside.
"""
import math

import numpy as np
import torch

own = False

E4M3, M4E3 = (4, 3), (3, 4)      # exponent and mantissa bits
EPS = 1e-5
_TYPES = {"float32": torch.float32, "bfloat16": torch.bfloat16, "codes": torch.uint8}


def _case(kind, name=None, **kw):
    c = {"kind": kind}
    if name is not None:
        c["name"] = name
    c.update(kw)
    return c


def _ln(name=None, **kw):
    return _case("layernorm", name, **{"x": "float32", "out": "codes", "train": False, **kw})


def _drop(name=None, **kw):
    return _case("dropout", name, **{"x": "float32", "out": "float32", "p": 0.1, "act": "none", "bias": True, "residual": True, "train": False, **kw})


def _dense(kind="dense", name=None, **kw):
    return _case(kind, name, **{"fmt": "e4m3", "acts": "normal", "act": "none", "bias": True, "residual": False, "p": 0.0, "out": "bfloat16",
                                "train": False, **kw})


def listed():
    return [
        # one new token between two layers: the row goes straight to the codes of the next product; latency is what counts
        _ln("layernorm_token_1x768", M=1, N=768),
        # a training step of the norm in a BERT-base layer, batch 32 of 128 tokens: forward to codes, backward of all three inputs
        _ln("layernorm_train_4096x768", M=4096, N=768, train=True),
        # the same on a wide model in bfloat16, where bandwidth is all there is
        _ln("layernorm_train_16384x4096_bf16", M=16384, N=4096, x="bfloat16", out="bfloat16", train=True),
        # what follows the attention's output product in training: float32 sums of a simulated product, scaled back, bias, dropout, residual
        _drop("dropout_4096x768", M=4096, N=768),
        # dropout behind the activation of a wide feed-forward layer, forward and backward, in bfloat16, with ragged sizes
        _drop("dropout_train_16411x4099_bf16", M=16411, N=4099, x="bfloat16", out="bfloat16", act="gelu", residual=False, train=True),
        # one token through a linear layer: a pass over the weights
        _dense(name="dense_token_1x4096x4096", M=1, N=4096, K=4096, residual=True),
        # the query, key and value product of a BERT-base layer, straight to bfloat16
        _dense(name="dense_qkv_4096x2304x768", M=4096, N=2304, K=768),
        # a training step of a ragged layer in float32: activation, dropout and residual in the epilogue, gradients of all inputs
        _dense(name="dense_train_3985x770x771", M=3985, N=770, K=771, act="gelu", residual=True, p=0.1, out="float32", train=True),
        # a large projection, activation and codes for the next product
        _dense(name="dense_8192x8192x4096", M=8192, N=8192, K=4096, act="gelu", out="codes"),
        # the paper's own operand format, M4E3 with flex bias, on the shape of a late ResNet-50 layer
        _dense(name="dense_m4e3_3136x512x4608", M=3136, N=512, K=4608, fmt="m4e3", acts="relu", act="relu"),
        # a few sequences that each add one token: the gated block's two projections in one pass over their weights
        _dense("gated", "gated_tokens_6x4096x2048", M=6, N=4096, K=2048, act="silu", bias=False, out="codes"),
        # a training step of the gated block
        _dense("gated", "gated_train_4096x4096x1024_bf16", M=4096, N=4096, K=1024, act="silu", bias=False, train=True),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(lo * (hi / lo) ** rng.random()))


def draw(rng):
    """One more case: any operator, sizes over the logarithm of their ranges, half of them of no round size."""
    kind = rng.choice(["layernorm", "dropout", "dense", "dense", "gated"])
    train = rng.random() < 0.5
    even = rng.random() < 0.5
    size = lambda lo, hi, step: max(step, _log_uniform(rng, lo, hi) // step * step) if even else _log_uniform(rng, lo, hi)  # noqa: E731
    if kind in ("layernorm", "dropout"):
        x = rng.choice(["float32", "bfloat16"])
        while True:
            M, N = _log_uniform(rng, 1, 16384), size(64, 8192, 64)
            if M * N <= (16384 * 2048 if x == "float32" else 16384 * 4096):
                break
        if kind == "layernorm":
            return _ln(M=M, N=N, x=x, out=rng.choice(["codes", x]), train=train)
        act = rng.choice(["none", "none", "relu", "gelu", "silu"])
        return _drop(M=M, N=N, x=x, out=x, p=rng.choice([0.05, 0.1, 0.1, 0.2, 0.5]), act=act, bias=rng.random() < 0.7,
                     residual=rng.random() < 0.6, train=train)
    while True:
        M = size(64, 8192, 64) if train or rng.random() < 0.6 else rng.randint(1, 48)
        N, K = size(96, 8192, 32), size(64, 4608, 32)
        macs = M * N * K * (2 if kind == "gated" else 1) * (3 if train else 1)
        if macs <= 8192 * 8192 * 2048:
            break
    out = rng.choice(["float32", "bfloat16"] if train else ["float32", "bfloat16", "codes"])
    act = rng.choice(["silu", "gelu", "relu"] if kind == "gated" else ["none", "none", "relu", "gelu", "silu"])
    return _dense(kind, M=M, N=N, K=K, fmt=rng.choice(["e4m3", "e4m3", "m4e3"]), acts=rng.choice(["normal", "relu"]), act=act,
                  bias=rng.random() < 0.6, residual=out != "codes" and rng.random() < 0.5, p=rng.choice([0.0, 0.1]) if train else 0.0,
                  out=out, train=train)


# ---- inputs ---------------------------------------------------------------------------------

def _values(E, M):
    """The 256 values of an 8-bit format at its canonical bias, every code a number."""
    c = np.arange(256)
    e, m, s = (c >> M) & ((1 << E) - 1), c & ((1 << M) - 1), np.where(c & 128, -1.0, 1.0)
    b = (1 << (E - 1)) - 1
    return s * np.where(e > 0, (1 + m / 2.0 ** M) * 2.0 ** (e - b), m * 2.0 ** (1 - b - M))


def _to_codes(x, E, M):
    """float32 tensor -> codes at the largest exponent bias that keeps its maximum inside the format, and that bias."""
    top = 448.0 if (E, M) == E4M3 else float(_values(E, M).max())
    t = math.floor(math.log2(top / float(x.abs().max())))
    grid = torch.from_numpy(_values(E, M)[:128].astype(np.float32)).to(x.device)
    mids = (grid[1:] + grid[:-1]) / 2
    code = torch.bucketize((x.abs() * 2.0 ** t).clamp(max=top), mids)
    return (code + 128 * (x < 0)).to(torch.uint8), (1 << (E - 1)) - 1 + t


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed) + 1)
    normal = lambda *shape: torch.randn(*shape, generator=g, device="cuda")  # noqa: E731
    kind, M, N = case["kind"], case["M"], case["N"]
    s = {"case": case, "seed": int(seed), "stream": 3 + 2 * int(seed)}
    t = torch.bfloat16 if "bfloat16" in (case.get("x", ""), case["out"]) else torch.float32
    if case["train"]:
        s["G"] = (normal(M, N) * 2.0 ** -8).to(t)
    if kind == "layernorm":
        s["x"] = (normal(M, N) * 1.7 + normal(N) * 0.3).to(_TYPES[case["x"]])
        s["gamma"], s["beta"] = 1 + 0.1 * normal(N), 0.1 * normal(N)
        s["fmt"] = (4, 3, 7 + 5)                       # eight times the deviation still fits
        return s
    if case["residual"]:
        s["residual"] = normal(M, N).to(t)
    if kind == "dropout":
        s["scale"] = 2.0 ** -9                          # of a product in code units
        s["x"] = (normal(M, N) * 2.0 ** 9).to(_TYPES[case["x"]])
        if case["bias"]:
            s["bias"] = 0.1 * normal(N)
        return s
    K, two = case["K"], 2 if kind == "gated" else 1
    E, m = E4M3 if case["fmt"] == "e4m3" else M4E3
    a = normal(M, K)
    s["A"], ba = _to_codes(a.clamp(min=0.0) if case["acts"] == "relu" else a, E, m)
    s["B"], bb = _to_codes(normal(two * N, K) * (1.5 / K) ** 0.5, E, m)
    s["fmt_a"], s["fmt_b"], s["fmt"] = (E, m, ba), (E, m, bb), (4, 3, 7 + 4)
    if case["bias"]:
        s["bias"] = 0.1 * normal(two * N)
    return s


# ---- the calls ------------------------------------------------------------------------------

def _run_own(s):
    from paper_2401_14110_amd import binding as lba
    case = s["case"]
    kind, out = case["kind"], _TYPES[case["out"]]
    fmt = s["fmt"] if case["out"] == "codes" else None
    shown = lambda y: y.view(torch.float8_e4m3fn) if fmt else y  # noqa: E731
    if kind == "layernorm":
        if not case["train"]:
            return {"y": shown(lba.layernorm(s["x"], s["gamma"], s["beta"], EPS, out_dtype=out, out_fmt=fmt))}
        y, mean, rstd = lba.layernorm(s["x"], s["gamma"], s["beta"], EPS, out_dtype=out, out_fmt=fmt, want_stats=True)
        dx, dgamma, dbeta = lba.layernorm_bwd(s["G"], s["x"], s["gamma"], mean, rstd)
        return {"y": shown(y), "dx": dx, "dgamma": dgamma, "dbeta": dbeta}
    act = {"none": lba.ACT_NONE, "relu": lba.ACT_RELU, "gelu": lba.ACT_GELU, "silu": lba.ACT_SILU}[case["act"]]
    drop = (case["p"], s["seed"], s["stream"]) if case["p"] > 0 else None
    bias, residual = s.get("bias"), s.get("residual")
    if kind == "dropout":
        y = lba.dropout(s["x"], drop, bias=bias, act=act, residual=residual, scale=s["scale"], out_dtype=out)
        if not case["train"]:
            return {"y": y}
        dx, dbias = lba.dropout_bwd(s["G"], drop, x=s["x"], bias=bias, act=act, scale=s["scale"], want_dbias=case["bias"])
        return {"y": y, "dx": dx, "dbias": dbias}
    gated = kind == "gated"
    y = lba.dense(s["A"], s["B"], s["fmt_a"], s["fmt_b"], bias=bias, act=act, residual=residual, drop=drop, gated=gated, out_dtype=out, out_fmt=fmt)
    if not case["train"]:
        return {"y": shown(y)}
    dA, dB, dbias = lba.dense_bwd(s["G"], s["A"], s["B"], s["fmt_a"], s["fmt_b"], bias=bias, act=act, drop=drop, gated=gated,
                                  want_dbias=case["bias"])
    return {"y": y, "dA": dA, "dB": dB, "dbias": dbias}


def _decoded(codes, fmt):
    E, M, b = fmt
    return torch.from_numpy((_values(E, M) * 2.0 ** ((1 << (E - 1)) - 1 - b)).astype(np.float32)).to(codes.device)[codes.long()]


def _act(z, act):
    if act == "relu":
        return z.clamp(min=0.0)
    if act == "gelu":
        return 0.5 * z * (1 + torch.erf(z * 0.7071067811865476))
    return z / (1 + torch.exp(-z)) if act == "silu" else z


def _act_slope(z, act):
    if act == "relu":
        return (z > 0).float()
    if act == "gelu":
        return 0.5 * (1 + torch.erf(z * 0.7071067811865476)) + z * torch.exp(-0.5 * z * z) * 0.3989422804014327
    if act == "silu":
        h = 1 / (1 + torch.exp(-z))
        return h * (1 + z * (1 - h))
    return torch.ones_like(z)


def _signed(v):
    v &= (1 << 64) - 1
    return v - (1 << 64) if v >> 63 else v


def _mixed(z):
    z &= (1 << 64) - 1
    z = (z ^ (z >> 30)) * 0xBF58476D1CE4E5B9 & ((1 << 64) - 1)
    z = (z ^ (z >> 27)) * 0x94D049BB133111EB & ((1 << 64) - 1)
    return z ^ (z >> 31)


_GOLDEN = 0x9E3779B97F4A7C15


def _base(s):
    return _mixed(_mixed(s["seed"] * 2 + 1) ^ ((s["stream"] * 2 + 1) * _GOLDEN))


def _threshold(p):
    return math.floor(p * 65536 + 0.5)


def _kept(s, M, N):
    """1 / (1 - p) where the value stays and 0 where it is dropped: 16 bits of a word of the counter-based generator for each element."""
    thr = _threshold(s["case"]["p"])
    i = torch.arange(M * N, device="cuda")
    right = lambda z, n: (z >> n) & ((1 << (64 - n)) - 1)  # noqa: E731
    z = (i >> 2) * _signed(_GOLDEN) + _signed(_base(s))
    z = (z ^ right(z, 30)) * _signed(0xBF58476D1CE4E5B9)
    z = (z ^ right(z, 27)) * _signed(0x94D049BB133111EB)
    z = z ^ right(z, 31)
    u = (z >> ((i & 3) * 16)) & 0xFFFF
    return torch.where(u >= thr, 65536.0 / (65536 - thr), 0.0).view(M, N)


def _coded(y, fmt):
    return (y * 2.0 ** (fmt[2] - 7)).clamp(-448.0, 448.0).to(torch.float8_e4m3fn)


def _out(s, y):
    return _coded(y, s["fmt"]) if s["case"]["out"] == "codes" else y.to(_TYPES[s["case"]["out"]])


def _run_plain(s):
    case = s["case"]
    kind, M, N = case["kind"], case["M"], case["N"]
    if kind == "layernorm":
        x = s["x"].float()
        c = x - x.mean(-1, keepdim=True)
        rstd = 1 / torch.sqrt((c * c).mean(-1, keepdim=True) + EPS)
        n = c * rstd
        y = _out(s, n * s["gamma"] + s["beta"])
        if not case["train"]:
            return {"y": y}
        G = s["G"].float()
        h = G * s["gamma"]
        dx = rstd * (h - h.mean(-1, keepdim=True) - n * (h * n).mean(-1, keepdim=True))
        return {"y": y, "dx": dx.to(s["x"].dtype), "dgamma": (G * n).sum(0), "dbeta": G.sum(0)}
    kept = _kept(s, M, N) if case["p"] > 0 else None
    if kind == "dropout":
        z = s["x"].float() * s["scale"]
    else:
        a, b = _decoded(s["A"], s["fmt_a"]), _decoded(s["B"], s["fmt_b"])
        z = a @ b.t()
    if "bias" in s:
        z = z + s["bias"]
    if kind == "gated":
        y = _act(z[:, :N], case["act"]) * z[:, N:]
    else:
        y = _act(z, case["act"])
    if kept is not None:
        y = y * kept
    if "residual" in s:
        y = y + s["residual"].float()
    y = _out(s, y)
    if not case["train"]:
        return {"y": y}
    d = s["G"].float()
    if kept is not None:
        d = d * kept
    if kind == "gated":
        d = torch.cat([d * z[:, N:] * _act_slope(z[:, :N], case["act"]), d * _act(z[:, :N], case["act"])], 1)
    else:
        d = d * _act_slope(z, case["act"])
    dbias = d.sum(0) if case["bias"] else None
    if kind == "dropout":
        return {"y": y, "dx": (d * s["scale"]).to(s["x"].dtype), "dbias": dbias}
    t = s["G"].dtype
    return {"y": y, "dA": (d @ b).to(t), "dB": (d.t() @ a).to(t), "dbias": dbias}


def run(s):
    return _run_own(s) if own else _run_plain(s)


# ---- the same in 64 bits --------------------------------------------------------------------

def _grid(v):
    """float64 -> the nearest value of E4M3, ties to the even code, at most 448."""
    v = v.clamp(-448.0, 448.0)
    q = torch.exp2(torch.floor(torch.log2(v.abs().clamp(min=2.0 ** -6))).clamp(min=-6.0) - 3)
    return torch.round(v / q) * q


def exact(case, seed):
    s = prepare(case, seed)
    f = torch.float64
    kind, M, N = case["kind"], case["M"], case["N"]
    res = {}

    def put(y):
        res["y"] = _grid(y * 2.0 ** (s["fmt"][2] - 7)) if case["out"] == "codes" else y

    if kind == "layernorm":
        x, gamma = s["x"].to(f), s["gamma"].to(f)
        var, mean = torch.var_mean(x, -1, correction=0, keepdim=True)
        sigma = (var + EPS) ** 0.5
        put((x - mean) / sigma * gamma + s["beta"].to(f))
        if case["train"]:
            G = s["G"].to(f)
            u = (x - mean) / sigma
            w = G * gamma
            res["dx"] = (N * w - w.sum(-1, keepdim=True) - u * (w * u).sum(-1, keepdim=True)) / (N * sigma)
            res["dgamma"], res["dbeta"] = torch.einsum("ij,ij->j", G, u), G.sum(0)
        return res
    keep = None
    if case["p"] > 0:
        with np.errstate(over="ignore"):
            w = np.arange((M * N + 3) // 4, dtype=np.uint64) * np.uint64(_GOLDEN) + np.uint64(_base(s))
            w = (w ^ (w >> np.uint64(30))) * np.uint64(0xBF58476D1CE4E5B9)
            w = (w ^ (w >> np.uint64(27))) * np.uint64(0x94D049BB133111EB)
            w ^= w >> np.uint64(31)
        thr = _threshold(case["p"])
        keep = torch.from_numpy((w.view(np.uint16)[:M * N] >= thr).reshape(M, N)).cuda().to(f) / (1 - thr / 65536)
    if kind == "dropout":
        z = s["x"].to(f) * s["scale"]
    else:
        val = lambda c, fmt: torch.from_numpy(_values(*fmt[:2])).cuda()[c.long()] * 2.0 ** ((1 << (fmt[0] - 1)) - 1 - fmt[2])  # noqa: E731
        a, b = val(s["A"], s["fmt_a"]), val(s["B"], s["fmt_b"])
        z = torch.matmul(a, b.t().contiguous())
    if case["bias"]:
        z = z + s["bias"].to(f)
    z.requires_grad_(True)
    v, up = (z[:, :N], z[:, N:]) if kind == "gated" else (z, None)
    if case["act"] == "relu":
        y = torch.where(v > 0, v, torch.zeros((), dtype=f, device="cuda"))
    elif case["act"] == "gelu":
        y = v * torch.special.ndtr(v)
    elif case["act"] == "silu":
        y = v * torch.sigmoid(v)
    else:
        y = v * 1.0
    if up is not None:
        y = y * up
    if keep is not None:
        y = y * keep
    if case["residual"]:
        y = y + s["residual"].to(f)
    put(y.detach())
    if case["train"]:
        (d,) = torch.autograd.grad(y, z, s["G"].to(f))
        if kind == "dropout":
            res["dx"] = d * s["scale"]
        else:
            res["dA"], res["dB"] = torch.matmul(d, b), torch.matmul(d.t().contiguous(), a)
        res["dbias"] = d.sum(0) if case["bias"] else None
    return res


# ---- what a pass cannot do without ----------------------------------------------------------

def work(case):
    """Each input read once and each output written once; a multiply-add of a product is two operations, an element of the others a few."""
    size = lambda t: {"float32": 4, "bfloat16": 2, "codes": 1}[t]  # noqa: E731
    kind, M, N, train = case["kind"], case["M"], case["N"], case["train"]
    grad = 2 if "bfloat16" in (case.get("x", ""), case["out"]) else 4
    y = M * N * size(case["out"])
    if kind == "layernorm":
        x = M * N * size(case["x"])
        return {"bytes": x + y + 8 * N + ((x + x + M * N * grad + 8 * N) if train else 0), "flops": M * N * (20 if train else 8)}
    extra = M * N * grad if case["residual"] else 0
    if kind == "dropout":
        x = M * N * size(case["x"])
        return {"bytes": x + y + extra + ((x + x + M * N * grad) if train else 0), "flops": M * N * (20 if train else 10)}
    K, two = case["K"], 2 if kind == "gated" else 1
    codes = M * K + two * N * K
    return {"bytes": codes + y + extra + ((codes * (1 + grad) + M * N * grad) if train else 0),
            "flops": 2.0 * M * N * K * two * (3 if train else 1)}

"""Layer norm and its gradients against the formulas in 64 bits, at the widths where lanes, vectors and workgroups end, for every type,
with rows that start anywhere; differences of the forward call; what must not leak between rows; refusals."""
import ctypes

import numpy as np
import pytest
import torch

import layer_oracle as lo
from paper_2401_14110_amd import binding as lb

DEV = "cuda:0"
DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def values(rng, shape, dtype, scale=1.0, offset=0.0):
    x = (rng.standard_normal(shape) * scale + offset).astype(np.float32)
    return lo.bf16(x) if dtype == "bf16" else x


def dev(x, dtype=None):
    t = torch.from_numpy(np.ascontiguousarray(x)).to(DEV)
    return t if dtype is None else t.to(DT[dtype])


def host(t):
    return t.float().cpu().numpy().astype(np.float64)


def near(got, want, tol, dtype):
    bound = tol + (2.0 ** -8 * np.abs(want) if dtype == "bf16" else 0.0)     # a bfloat16 result is rounded once: 2^-9, and once more of the error
    bad = np.abs(host(got) - want) > bound
    assert not bad.any(), (int(bad.sum()), np.argwhere(bad)[:3], host(got)[bad][:3], want[bad][:3])


WIDTHS = [1, 2, 3, 7, 8, 63, 64, 65, 255, 256, 257, 511, 770, 1023, 1024, 1025, 2047, 2049, 4096, 4099, 8191, 8200, 16384]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("N", WIDTHS)
def test_forward_and_gradients(N, dtype):
    rng = np.random.default_rng(N)
    for M in (1, 5) if N > 3000 else (1, 4, 37):
        x, G = values(rng, (M, N), dtype, 2.0, 0.5), values(rng, (M, N), dtype)
        gamma, beta = values(rng, N, "f32", 0.2, 1.0), values(rng, N, "f32", 0.3)
        y64, mean, rstd, tol = lo.norm(x.astype(np.float64), gamma.astype(np.float64), beta.astype(np.float64), 1e-5)
        tx, tg, tb = dev(x, dtype), dev(gamma), dev(beta)
        y, m, r = lb.layernorm(tx, tg, tb, want_stats=True)
        assert y.dtype == DT[dtype]
        near(y, y64, tol, dtype)
        near(m, mean, (64 + N / 512) * lo.U * np.abs(x).mean(-1).astype(np.float64) + 1e-37, "f32")
        dx, dgamma, dbeta = lb.layernorm_bwd(dev(G, dtype), tx, tg, m, r)
        want, tols = lo.norm_bwd(G.astype(np.float64), x.astype(np.float64), gamma.astype(np.float64), host(m), host(r))
        near(dx, want[0], tols[0], dtype)
        near(dgamma, want[1], tols[1], "f32")
        near(dbeta, want[2], tols[2], "f32")


@pytest.mark.gpu
@pytest.mark.parametrize("N", [5, 768, 1030, 4100, 20000])
@pytest.mark.parametrize("fmt", [(4, 3, 11), (3, 4, 6), (5, 2, 15), (2, 5, 4), (4, 3, -3)])
def test_codes_out(N, fmt):
    rng = np.random.default_rng(N + fmt[2])
    for dtype in ("f32", "bf16"):
        x = values(rng, (9, N), dtype, 3.0, -1.0)
        y64, _, _, tol = lo.norm(x.astype(np.float64), None, None, 1e-5)
        codes = lb.layernorm(dev(x, dtype), out_dtype=torch.uint8, out_fmt=fmt)
        assert codes.dtype == torch.uint8
        lo.check_codes(codes.cpu().numpy(), y64, tol, fmt)


@pytest.mark.gpu
@pytest.mark.parametrize("M,N", [(4096, 768), (700, 4100), (300, 16384)])
@pytest.mark.parametrize("fmt", [(4, 3, 12), (3, 4, 6)])
def test_codes_are_the_nearest(M, N, fmt):
    """Rows that stay in registers: the code of every element is that of the exact value, also next to the middle of two codes."""
    rng = np.random.default_rng(M)
    x, g, b = values(rng, (M, N), "f32", 2.0, 0.5), values(rng, N, "f32", 0.3, 1.0), values(rng, N, "f32", 0.2)
    y64, _, _, _ = lo.norm(x.astype(np.float64), g.astype(np.float64), b.astype(np.float64), 1e-5)
    codes = lb.layernorm(dev(x), dev(g), dev(b), 1e-5, out_dtype=torch.uint8, out_fmt=fmt).cpu().numpy()
    near64 = lo.nearest_code_value(y64, *fmt)
    off = lo.code_values(*fmt)[codes] != near64
    assert off.sum() == 0, (int(off.sum()), y64[off][:4], near64[off][:4])


@pytest.mark.gpu
@pytest.mark.parametrize("N", [64, 770, 16384, 20000])
def test_results_beyond_float32_saturate(N):
    rng = np.random.default_rng(N)
    x, g = values(rng, (40, N), "f32"), np.where(np.arange(N) % 2, 3e38, -1e38).astype(np.float32)
    y64, _, _, _ = lo.norm(x.astype(np.float64), g.astype(np.float64), None, 1e-5)
    assert (np.abs(y64) > 3.5e38).any() and (np.abs(y64) > 1e30).all()
    for fmt in ((4, 3, 7), (3, 4, 3), (5, 2, 15)):
        codes = lb.layernorm(dev(x), dev(g), out_dtype=torch.uint8, out_fmt=fmt).cpu().numpy()
        assert np.array_equal(codes, np.where(y64 < 0, 0x80, 0) + (0x7E if fmt[0] == 4 else 0x7F))
    # infinities of the parameters saturate, and NaN stays NaN
    beta = np.zeros(N, np.float32)
    beta[1], beta[2], beta[3] = np.inf, -np.inf, np.nan
    codes = lb.layernorm(dev(x), None, dev(beta), out_dtype=torch.uint8, out_fmt=(4, 3, 7)).cpu().numpy()
    assert (codes[:, 1] == 0x7E).all() and (codes[:, 2] == 0xFE).all() and (codes[:, 3] & 0x7F == 0x7F).all()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("N", [16385, 70001])
def test_rows_beyond_the_registers(N, dtype):
    rng = np.random.default_rng(N)
    x, G, gamma = values(rng, (3, N), dtype), values(rng, (3, N), dtype), values(rng, N, "f32", 0.2, 1.0)
    y64, _, _, tol = lo.norm(x.astype(np.float64), gamma.astype(np.float64), None, 1e-3)
    y, m, r = lb.layernorm(dev(x, dtype), dev(gamma), eps=1e-3, want_stats=True)
    near(y, y64, tol, dtype)
    dx, dgamma, dbeta = lb.layernorm_bwd(dev(G, dtype), dev(x, dtype), dev(gamma), m, r)
    want, tols = lo.norm_bwd(G.astype(np.float64), x.astype(np.float64), gamma.astype(np.float64), host(m), host(r))
    near(dx, want[0], tols[0], dtype)
    near(dgamma, want[1], tols[1], "f32")
    near(dbeta, want[2], tols[2], "f32")


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_many_rows_beyond_the_registers(dtype):
    """More rows than the launch has workgroups: a row's result does not depend on the rows that its workgroup has before and after it."""
    M, N, part = 150001, 16400, 60000                            # a call of `part` rows gives each of them a workgroup
    gen = torch.Generator(device=DEV).manual_seed(1)
    x, G = (torch.randn(M, N, generator=gen, device=DEV).to(DT[dtype]) for _ in range(2))
    x *= 1 + torch.arange(M, device=DEV).view(-1, 1) % 7         # another row's sums would show
    gamma = torch.randn(N, generator=gen, device=DEV)
    y, m, r = lb.layernorm(x, gamma, want_stats=True)
    dx, _, _ = lb.layernorm_bwd(G, x, gamma, m, r, want_params=False)
    for k in range(0, M, part):
        s = slice(k, k + part)
        one = lb.layernorm(x[s], gamma, want_stats=True)
        assert torch.equal(one[0], y[s]) and torch.equal(one[1], m[s]) and torch.equal(one[2], r[s]), k
        assert torch.equal(lb.layernorm_bwd(G[s], x[s], gamma, m[s], r[s], want_params=False)[0], dx[s]), k


@pytest.mark.gpu
@pytest.mark.parametrize("M", [1023, 4097, 20011])
def test_many_rows(M):
    # more rows than workgroups write partial sums for
    rng = np.random.default_rng(M)
    for N, dtype in ((70, "f32"), (1040, "bf16"), (2052, "f32")):
        x, G = values(rng, (M, N), dtype), values(rng, (M, N), dtype)
        m = x.astype(np.float64).mean(-1).astype(np.float32)
        r = (1 / np.sqrt(x.astype(np.float64).var(-1) + 1e-5)).astype(np.float32)
        want, tols = lo.norm_bwd(G.astype(np.float64), x.astype(np.float64), None, m.astype(np.float64), r.astype(np.float64))
        tG, tx = dev(G, dtype), dev(x, dtype)
        dx, dgamma, dbeta = lb.layernorm_bwd(tG, tx, None, dev(m), dev(r))
        near(dx, want[0], tols[0], dtype)
        near(dgamma, want[1], tols[1], "f32")
        near(dbeta, want[2], tols[2], "f32")
        again = lb.layernorm_bwd(tG, tx, None, dev(m), dev(r))
        assert torch.equal(again[1], dgamma) and torch.equal(again[2], dbeta)      # the same bits on every run
        only = lb.layernorm_bwd(tG, tx, None, dev(m), dev(r), want_dx=False)
        assert only[0] is None and torch.equal(only[1], dgamma)
        assert torch.equal(lb.layernorm_bwd(tG, tx, None, dev(m), dev(r), want_params=False)[0], dx)


@pytest.mark.gpu
def test_mixed_types_strides_and_leading_axes():
    rng = np.random.default_rng(5)
    for gt, xt in (("f32", "bf16"), ("bf16", "f32")):
        x, G = values(rng, (6, 300), xt), values(rng, (6, 300), gt)
        y, m, r = lb.layernorm(dev(x, xt), want_stats=True)
        dx, dgamma, _ = lb.layernorm_bwd(dev(G, gt), dev(x, xt), None, m, r)
        want, tols = lo.norm_bwd(G.astype(np.float64), x.astype(np.float64), None, host(m), host(r))
        assert dx.dtype == DT[xt]
        near(dx, want[0], tols[0], xt)
        near(dgamma, want[1], tols[1], "f32")
    # rows off every alignment, a transposed view, three axes
    base = dev(values(rng, 1 + 7 * 129, "f32"))
    x = base[1:].view(7, 129)
    want, _, _, tol = lo.norm(host(x), None, None, 1e-5)
    near(lb.layernorm(x), want, tol, "f32")
    t = dev(values(rng, (130, 12), "bf16"), "bf16").t()
    want, _, _, tol = lo.norm(host(t), None, None, 1e-5)
    near(lb.layernorm(t), want, tol, "bf16")
    z = dev(values(rng, (2, 3, 40), "f32"))
    y, m, r = lb.layernorm(z, want_stats=True)
    assert y.shape == z.shape and m.shape == (2, 3)
    want, _, _, tol = lo.norm(host(z), None, None, 1e-5)
    near(y, want, tol, "f32")


@pytest.mark.gpu
def test_differences():
    # the loss sum(G * y) along a direction: central differences of the forward call against the gradients
    rng = np.random.default_rng(8)
    M, N, eps = 6, 96, 2.0 ** -7
    x, G, gamma, beta = (rng.standard_normal(s) for s in ((M, N), (M, N), N, N))
    loss = lambda x, g, b: float((G * host(lb.layernorm(dev(x.astype(np.float32)), dev(g.astype(np.float32)), dev(b.astype(np.float32))))).sum())  # noqa: E731
    x, gamma, beta = (a.astype(np.float32).astype(np.float64) for a in (x, gamma, beta))
    y, m, r = lb.layernorm(dev(x.astype(np.float32)), dev(gamma.astype(np.float32)), dev(beta.astype(np.float32)), want_stats=True)
    grads = [host(t) for t in lb.layernorm_bwd(dev(G.astype(np.float32)), dev(x.astype(np.float32)), dev(gamma.astype(np.float32)), m, r)]
    for k, arg in enumerate((x, gamma, beta)):
        v = np.sign(rng.standard_normal(arg.shape))
        up, down = [[a + (s * eps * v if i == k else 0) for i, a in enumerate((x, gamma, beta))] for s in (1, -1)]
        slope = (loss(*up) - loss(*down)) / (2 * eps)
        # third-order error eps^2 of terms of size |G| in number M * N, added at random: below 1e-2 of the scale sqrt(M N); float32 noise is less
        assert abs(slope - float((grads[k] * v).sum())) <= 1e-2 * np.sqrt(M * N), k


@pytest.mark.gpu
def test_rows_stay_apart_and_constant_rows():
    x = torch.randn(5, 600, device=DEV)
    clean = lb.layernorm(x)
    x2 = x.clone()
    x2[1, 7] = float("nan")
    x2[3, 599] = float("inf")
    y = lb.layernorm(x2)
    assert torch.equal(y[[0, 2, 4]], clean[[0, 2, 4]]) and y[1].isnan().all() and y[3].isnan().any()
    codes = lb.layernorm(x2, out_dtype=torch.uint8, out_fmt=(4, 3, 11))
    assert (codes[1] & 127 == 127).all()
    const = torch.full((3, 1000), 7.0, device=DEV)
    y, m, r = lb.layernorm(const, want_stats=True)
    assert (y == 0).all() and (m == 7).all()
    dx, dg, _ = lb.layernorm_bwd(torch.ones_like(const), const, None, m, r)
    assert dx.abs().max() <= 1e-3 * 2 ** -10 and (dg == 0).all()
    # a mean far above the deviation: nothing cancels
    far = torch.randn(4, 2048, device=DEV) + 4096
    want, _, _, tol = lo.norm(host(far), None, None, 1e-5)
    near(lb.layernorm(far), want, tol, "f32")


@pytest.mark.gpu
def test_in_place_side_streams_and_empty():
    x = torch.randn(300, 770, device=DEV)
    want = lb.layernorm(x)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    got = lb.layernorm(x, stream=s)
    t = lb.layernorm(torch.randn(770, 300, device=DEV).t(), stream=s)
    s.synchronize()
    assert torch.equal(got, want) and t.shape == (300, 770)
    y = x.clone()
    assert lb.layernorm(y, out=y) is y and torch.equal(y, want)
    assert lb.layernorm(torch.empty(0, 5, device=DEV)).shape == (0, 5)
    e = torch.empty(0, 5, device=DEV)
    z = torch.empty(0, device=DEV)
    _, dg, db = lb.layernorm_bwd(e, e, None, z, z)
    assert (dg == 0).all() and (db == 0).all()


@pytest.mark.gpu
def test_offsets_beyond_32_bits():
    M, N = (1 << 20) + 3, 4099                                   # 4.3e9 elements
    x = torch.zeros((M, N), dtype=torch.bfloat16, device=DEV)
    tail = torch.randn(3, N, device=DEV).bfloat16()
    x[-3:] = tail
    y, m, r = lb.layernorm(x, want_stats=True, out=x)
    want, _, _, tol = lo.norm(host(tail), None, None, 1e-5)
    near(y[-3:], want, tol, "bf16")
    assert (y[:5] == 0).all() and (m[-3:] != 0).all()
    g = x
    g[:-3] = 1
    src = torch.zeros_like(x)
    src[-3:] = tail
    dx, dg, db = lb.layernorm_bwd(g, src, None, m, r, want_dx=False)
    w = lo.norm_bwd(host(g[-3:]), host(tail), None, host(m[-3:]), host(r[-3:]))
    near(dg, w[0][1], w[1][1] + 64 * lo.U * np.abs(w[0][1]), "f32")
    assert ((db - (M - 3) - g[-3:].float().sum(0)).abs() <= 64).all()   # sums of ones to 2^20 are exact in parts; the last three are not


def test_refusals():
    P = ctypes.c_void_p(0x1000)
    W = ctypes.c_void_p(0x2000)
    f = (4, 3, 7)
    call = lambda **k: lb.lba_layernorm(*{**dict(X=P, x_type=0, g=None, b=None, eps=1e-5, Y=P, y_type=0, f=f, m=None, r=None, M=4, N=8), **k}.values())  # noqa: E731
    assert call(X=None) == lb.ERR_NULL and call(Y=None) == lb.ERR_NULL
    assert call(M=-1) == lb.ERR_SHAPE and call(N=(1 << 21) + 1) == lb.ERR_SHAPE and call(M=1 << 31) == lb.ERR_SHAPE
    assert call(x_type=2) == lb.ERR_UNSUPPORTED and call(y_type=3) == lb.ERR_UNSUPPORTED
    assert call(y_type=2, f=(6, 1, 7)) == lb.ERR_FORMAT and call(y_type=2, f=(4, 3, 33)) == lb.ERR_FORMAT
    assert call(M=0, X=None) == lb.OK and call(N=0) == lb.OK
    need = lb.lba_layernorm_bwd_workspace_bytes(4, 8)
    assert need > 0 and lb.lba_layernorm_bwd_workspace_bytes(0, 8) == 0
    back = lambda **k: lb.lba_layernorm_bwd(*{**dict(G=P, gt=0, X=P, xt=0, gamma=None, m=P, r=P, dX=P, dg=P, db=P, M=4, N=8, ws=W, n=need), **k}.values())  # noqa: E731
    assert back(G=None) == lb.ERR_NULL and back(m=None) == lb.ERR_NULL and back(dX=None, dg=None, db=None) == lb.ERR_NULL
    assert back(ws=None) == lb.ERR_NULL and back(n=need - 1) == lb.ERR_SHAPE and back(ws=ctypes.c_void_p(0x2010)) == lb.ERR_ALIGN
    assert back(gt=5) == lb.ERR_UNSUPPORTED and back(M=-2) == lb.ERR_SHAPE


def test_binding_refusals():
    with pytest.raises(TypeError):
        lb.layernorm(torch.zeros(2, 3))                          # not on the device

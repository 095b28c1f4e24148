"""Dropout with bias, activation and residual, and its gradients, against the formulas and the generator in 64 bits: widths where strips,
tails and words of the generator end, every type, rates from none to all, the step word, replays of a captured graph; refusals."""
import ctypes

import numpy as np
import pytest
import torch

import layer_oracle as lo
from paper_2401_14110_amd import binding as lb
from test_gpu_layernorm import DEV, dev, host, near, values

ACT_TOL = 16 * lo.U                  # relative to |z| + |act(z)|: a few roundings of the argument and of erf or exp


def forward(x, bias, residual, scale, act, f):
    z = x * scale + (0 if bias is None else bias)
    v, slope = lo.act(z, act)
    y = np.where(f != 0, v * f, 0.0) + (0 if residual is None else residual)
    tol = ACT_TOL * ((np.abs(x * scale) + (0 if bias is None else np.abs(bias))) * 1.2 * (f + 1) + np.abs(y) + (0 if residual is None else np.abs(residual))) + 1e-37
    return z, slope, y, tol


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("N", [1, 2, 3, 5, 8, 63, 64, 129, 255, 256, 257, 512, 513, 770, 1023, 1540, 4099])
def test_forward_and_gradients(N, dtype):
    rng = np.random.default_rng(N)
    for k, M in enumerate((1, 3, 66, 517)):
        act, p, seed, stream = (N + k) % 4, (0.1, 0.5, 0.0, 0.03)[k], N * 77 + k, 2 ** 63 + N
        x, G, R = (values(rng, (M, N), dtype, s) for s in (8.0, 1.0, 1.0))
        b = values(rng, N, "f32", 0.5) if k != 1 else None
        scale = 0.25
        f = lo.drop_factors(p, seed, stream, 0, M * N).reshape(M, N)
        z, slope, y64, tol = forward(x.astype(np.float64), b, R.astype(np.float64), scale, act, f)
        tx, tb = dev(x, dtype), (dev(b) if b is not None else None)
        y = lb.dropout(tx, (p, seed, stream), bias=tb, act=act, residual=dev(R, dtype), scale=scale)
        near(y, y64, tol, dtype)
        dx, db = lb.dropout_bwd(dev(G, dtype), (p, seed, stream), x=tx, bias=tb, act=act, scale=scale, want_dbias=True)
        d64 = G.astype(np.float64) * f * slope
        td = 40 * lo.U * np.abs(G) * f * (np.abs(z) + 1) + 1e-37                  # act'' is below 1.2, the argument is rounded twice
        near(dx, d64 * scale, td * scale, dtype)
        near(db, d64.sum(0), td.sum(0) + (M + 64) * lo.U * np.abs(d64).sum(0) + 1e-37, "f32")


@pytest.mark.gpu
def test_mask_is_the_generators_and_the_same_in_both_passes():
    for N in (64, 65, 770):
        x = torch.ones(200, N, device=DEV)
        y = lb.dropout(x, (0.3, 11, 5))
        f = lo.drop_factors(0.3, 11, 5, 0, 200 * N).reshape(200, N)
        assert np.array_equal(y.cpu().numpy(), f.astype(np.float32))
        assert torch.equal(lb.dropout_bwd(x, (0.3, 11, 5))[0], y)
        assert abs(float((y == 0).float().mean()) - 0.3) < 5 * (0.21 / (200 * N)) ** 0.5
        assert not torch.equal(lb.dropout(x, (0.3, 11, 6)), y) and not torch.equal(lb.dropout(x, (0.3, 12, 5)), y)
    bf = torch.ones(64, 512, device=DEV, dtype=torch.bfloat16)                    # the mask does not depend on the type
    assert torch.equal(lb.dropout(bf, (0.3, 1, 2)) != 0, lb.dropout(bf.float(), (0.3, 1, 2)) != 0)


@pytest.mark.gpu
@pytest.mark.parametrize("act", [lb.ACT_NONE, lb.ACT_RELU, lb.ACT_GELU, lb.ACT_SILU])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_masks_of_many_rows_that_end_inside_a_word(act, dtype):
    """Every bit of the mask, both passes, where the chip is full and the elements' bits are cut out of two words."""
    M, N = 8192, 4107
    x = torch.ones(M, N, device=DEV, dtype=torch.float32 if dtype == "f32" else torch.bfloat16)
    keep = torch.from_numpy(lo.drop_factors(0.5, 7, 3, 0, M * N).reshape(M, N) > 0).to(DEV)
    assert torch.equal(lb.dropout(x, (0.5, 7, 3), act=act) != 0, keep)
    assert torch.equal(lb.dropout_bwd(x, (0.5, 7, 3), x=x, act=act)[0] != 0, keep)


@pytest.mark.gpu
def test_rates_at_the_ends_and_values_that_are_dropped():
    x = torch.randn(33, 130, device=DEV)
    r = torch.randn(33, 130, device=DEV)
    assert torch.equal(lb.dropout(x, None), x) and torch.equal(lb.dropout(x, (0.0, 1, 1), residual=r), x + r)
    assert torch.equal(lb.dropout(x, (1.0, 1, 1), residual=r), r) and (lb.dropout_bwd(x, (1.0, 1, 1))[0] == 0).all()
    bad = x.clone()
    f = torch.from_numpy(lo.drop_factors(0.5, 3, 4, 0, 33 * 130).reshape(33, 130)).to(DEV)
    bad[f == 0] = float("nan")
    bad[5][f[5] == 0] = float("inf")
    y = lb.dropout(bad, (0.5, 3, 4), act=lb.ACT_GELU)
    assert y.isfinite().all() and torch.equal(y, lb.dropout(x, (0.5, 3, 4), act=lb.ACT_GELU))
    y = lb.dropout(torch.full((4, 8), float("nan"), device=DEV), None, act=lb.ACT_RELU)
    assert y.isnan().all()


@pytest.mark.gpu
@pytest.mark.parametrize("fmt", [(4, 3, 9), (3, 4, 5)])
def test_codes_and_mixed_types(fmt):
    rng = np.random.default_rng(4)
    for dtype, rt in (("f32", "bf16"), ("bf16", "f32")):
        x, R = values(rng, (40, 333), dtype, 300.0), values(rng, (40, 333), rt)
        f = lo.drop_factors(0.1, 9, 9, 0, 40 * 333).reshape(40, 333)
        _, _, y64, tol = forward(x.astype(np.float64), None, R.astype(np.float64), 2.0 ** -8, 3, f)
        codes = lb.dropout(dev(x, dtype), (0.1, 9, 9), act=lb.ACT_SILU, residual=dev(R, rt), scale=2.0 ** -8, out_dtype=torch.uint8, out_fmt=fmt)
        lo.check_codes(codes.cpu().numpy(), y64, tol, fmt)
        y = lb.dropout(dev(x, dtype), (0.1, 9, 9), act=lb.ACT_SILU, residual=dev(R, rt), scale=2.0 ** -8, out_dtype=torch.float32)
        near(y, y64, tol, "f32")


@pytest.mark.gpu
def test_step_word_and_graph_replays():
    x = torch.randn(257, 384, device=DEV)
    step = torch.zeros(1, dtype=torch.int64, device=DEV)
    for k in (0, 5, -3):
        step.fill_(k)
        assert torch.equal(lb.dropout(x, (0.2, 7, 100, step)), lb.dropout(x, (0.2, 7, 100 + k)))
    out, dx = torch.empty_like(x), None
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        lb.dropout(x, (0.2, 7, 100, step), out=out)
        lb.dropout_bwd(x, (0.2, 7, 100, step), want_dbias=True)
    torch.cuda.current_stream().wait_stream(s)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        lb.dropout(x, (0.2, 7, 100, step), out=out)
        dx, db = lb.dropout_bwd(x, (0.2, 7, 100, step), want_dbias=True)
    for k in range(4):
        step.fill_(k)
        x.copy_(torch.randn_like(x))
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, lb.dropout(x, (0.2, 7, 100 + k)))
        wx, wb = lb.dropout_bwd(x, (0.2, 7, 100 + k), want_dbias=True)
        assert torch.equal(dx, wx) and torch.equal(db, wb)


@pytest.mark.gpu
def test_activations_far_out():
    z = np.array([-3e38, -1e30, -1e4, -200.0, -104.0, -100.0, -90.0, -88.8, -88.73, -80.0, -20.0, -0.0, 0.0, 1e-30, 20.0, 88.0, 89.0, 1e4, 1e30, 3e38], np.float32)
    for act in (1, 2, 3):
        with np.errstate(over="ignore"):
            v, slope = lo.act(z.astype(np.float64), act)
        y = lb.dropout(dev(z), None, act=act)
        dx, _ = lb.dropout_bwd(torch.ones(20, device=DEV), None, x=dev(z), act=act)
        # 1 + erf cancels below zero: the error is that of the sum, relative to |z|; elsewhere a few roundings
        near(y, v, 16 * lo.U * (np.abs(v) + np.minimum(np.abs(z.astype(np.float64)), 6.0)) + 1e-37, "f32")
        near(dx, slope, 24 * lo.U * (np.abs(slope) + 1) + 1e-37, "f32")


@pytest.mark.gpu
def test_gelu_of_what_is_no_number():
    z = torch.tensor([float("inf"), float("-inf"), float("nan"), 1.0], device=DEV)
    y = lb.dropout(z, None, act=lb.ACT_GELU).cpu()
    assert y[0] == float("inf") and y[1] == 0 and y[2].isnan() and y[3].isfinite()
    dx = lb.dropout_bwd(torch.ones(4, device=DEV), None, x=z, act=lb.ACT_GELU)[0].cpu()
    assert dx[0] == 1 and dx[1] == 0 and dx[2].isnan() and dx[3].isfinite()
    code = lb.dropout(z, None, out_dtype=torch.uint8, out_fmt=(4, 3, 7)).cpu()
    assert code[:2].tolist() == [0x7E, 0xFE] and int(code[2]) in (0x7F, 0xFF) and code[3] == 0x38


@pytest.mark.gpu
def test_differences():
    rng = np.random.default_rng(12)
    M, N, eps = 16, 48, 2.0 ** -7
    x, G, b = rng.standard_normal((M, N)), rng.standard_normal((M, N)), rng.standard_normal(N)
    x, b = x.astype(np.float32), b.astype(np.float32)
    for act in (lb.ACT_GELU, lb.ACT_SILU):
        drop = (0.25, 3, 3)
        loss = lambda x, b: float((G * host(lb.dropout(dev(x), drop, bias=dev(b), act=act, scale=0.5))).sum())  # noqa: E731
        dx, db = lb.dropout_bwd(dev(G.astype(np.float32)), drop, x=dev(x), bias=dev(b), act=act, scale=0.5, want_dbias=True)
        for arg, grad in ((0, dx), (1, db)):
            v = np.sign(rng.standard_normal(x.shape if arg == 0 else b.shape)).astype(np.float32)
            step = np.float32(eps) * v
            args = [(x + s * step, b) if arg == 0 else (x, b + s * step) for s in (np.float32(1), np.float32(-1))]
            slope = (loss(*args[0]) - loss(*args[1])) / (2 * eps)
            # third-order error eps^2 of M N terms of size |G|, added at random: below 1e-2 of the scale sqrt(M N)
            assert abs(slope - float((host(grad) * v).sum())) <= 1e-2 * np.sqrt(M * N), (act, arg)


@pytest.mark.gpu
def test_views_streams_and_empty():
    base = torch.randn(1 + 9 * 201, device=DEV)
    x = base[1:].view(9, 201)
    assert torch.equal(lb.dropout(x, (0.4, 1, 1)), lb.dropout(x.clone(), (0.4, 1, 1)))
    t = torch.randn(64, 90, device=DEV).t()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    y = lb.dropout(t, (0.4, 1, 1), stream=s)
    s.synchronize()
    assert torch.equal(y, lb.dropout(t.contiguous(), (0.4, 1, 1)))
    z = t.contiguous()
    want = lb.dropout(z, (0.4, 1, 1))
    assert lb.dropout(z, (0.4, 1, 1), out=z) is z and torch.equal(z, want)
    e = torch.empty(0, 7, device=DEV)
    assert lb.dropout(e, (0.4, 1, 1)).shape == (0, 7) and (lb.dropout_bwd(e, (0.4, 1, 1), want_dbias=True)[1] == 0).all()


@pytest.mark.gpu
def test_offsets_beyond_32_bits():
    M, N = (1 << 20) + 3, 4099
    x = torch.ones((M, N), dtype=torch.bfloat16, device=DEV)
    y = lb.dropout(x, (0.5, 21, 22), out=x)
    start = (M - 3) * N
    f = lo.drop_factors(0.5, 21, 22, start, 3 * N).reshape(3, N)
    assert np.array_equal(host(y[-3:]), f)


def test_refusals():
    P, W, f = ctypes.c_void_p(0x1000), ctypes.c_void_p(0x2000), (4, 3, 7)
    d = lambda p: lb.lba_drop(p, 1, 2, None)  # noqa: E731
    call = lambda **k: lb.lba_dropout(*{**dict(X=P, xt=0, scale=1.0, bias=None, act=0, drop=d(0.1), R=None, rt=0, Y=P, yt=0, f=f, M=4, N=8), **k}.values())  # noqa: E731
    assert call(X=None) == lb.ERR_NULL and call(Y=None) == lb.ERR_NULL
    assert call(drop=d(-0.1)) == lb.ERR_FORMAT and call(drop=d(1.5)) == lb.ERR_FORMAT and call(drop=d(float("nan"))) == lb.ERR_FORMAT
    assert call(act=4) == lb.ERR_UNSUPPORTED and call(xt=2) == lb.ERR_UNSUPPORTED and call(R=P, rt=2) == lb.ERR_UNSUPPORTED
    assert call(M=-1) == lb.ERR_SHAPE and call(N=1 << 22) == lb.ERR_SHAPE and call(yt=2, f=(1, 6, 0)) == lb.ERR_FORMAT
    assert call(M=0) == lb.OK
    need = lb.lba_dropout_bwd_workspace_bytes(4, 8)
    back = lambda **k: lb.lba_dropout_bwd(*{**dict(G=P, gt=0, X=P, xt=0, scale=1.0, bias=None, act=2, drop=d(0.1), dX=P, db=P, M=4, N=8, ws=W, n=need), **k}.values())  # noqa: E731
    assert back(X=None) == lb.ERR_NULL and back(G=None) == lb.ERR_NULL and back(dX=None, db=None) == lb.ERR_NULL
    assert back(ws=None) == lb.ERR_NULL and back(n=need - 1) == lb.ERR_SHAPE and back(ws=ctypes.c_void_p(0x2001)) == lb.ERR_ALIGN
    assert back(drop=d(2.0)) == lb.ERR_FORMAT and back(act=-1) == lb.ERR_UNSUPPORTED

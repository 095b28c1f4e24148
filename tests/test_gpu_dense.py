"""The dense product of codes with its epilogue, the gated one, and their gradients, against the formulas in 64 bits: few rows and tiles of
every size, ends of rows, tiles and steps, all formats and types; differences; offsets; what the calls refuse."""
import ctypes

import numpy as np
import pytest
import torch

import layer_oracle as lo
from paper_2401_14110_amd import binding as lb
from test_gpu_layernorm import DEV, DT, dev, host, near, values

E4M3, M4E3, E5M2, E2M5 = (4, 3, 10), (3, 4, 5), (5, 2, 17), (2, 5, 3)


def codes(rng, shape, fmt):
    c = rng.integers(0, 256, shape).astype(np.uint8)
    if fmt[0] == 4:
        c = np.where((c & 127) > 0x70, c & 0xBF, c).astype(np.uint8)        # no NaN codes
    if fmt[0] == 5:
        c = (c & 0x9F) | 0x20                                               # a few binades around the bias
    return c.astype(np.uint8)


def problem(seed, M, N, K, fa, fb, gated, with_bias, dtype, with_residual, p):
    rng = np.random.default_rng(seed)
    two = 2 if gated else 1
    A, B = codes(rng, (M, K), fa), codes(rng, (two * N, K), fb)
    # sums of the size of activations: the formats' biases take the scale
    a, b = lo.code_values(*fa)[A[:64]], lo.code_values(*fb)[B[:64]]
    down = int(np.round(np.log2(max(1e-9, np.sqrt((a ** 2).mean() * (b ** 2).mean() * max(K, 1))))))
    fa = (fa[0], fa[1], min(32, fa[2] + down))
    bias = values(rng, two * N, "f32", 0.5) if with_bias else None
    R = values(rng, (M, N), dtype) if with_residual else None
    G = values(rng, (M, N), dtype)
    drop = (p, seed, 2 ** 40 + seed) if p else None
    f = lo.drop_factors(p, seed, 2 ** 40 + seed, 0, M * N).reshape(M, N) if p else None
    return A, B, fa, fb, bias, R, G, drop, f


def run(seed, M, N, K, fa=E4M3, fb=E4M3, gated=False, act=0, bias=True, residual=True, p=0.0, dtype="f32", train=True):
    A, B, fa, fb, b, R, G, drop, f = problem(seed, M, N, K, fa, fb, gated, bias, dtype, residual, p)
    opt = lambda t, d=None: None if t is None else dev(t, d)  # noqa: E731
    y64, tol, parts = lo.dense(A, B, fa, fb, None if b is None else b.astype(np.float64), act, gated, f, None if R is None else R.astype(np.float64))
    tA, tB, tb = dev(A), dev(B), opt(b)
    y = lb.dense(tA, tB, fa, fb, bias=tb, act=act, residual=opt(R, dtype), drop=drop, gated=gated, out_dtype=DT[dtype])
    near(y, y64, tol, dtype)
    if not train:
        return
    dA, dB, db = lb.dense_bwd(dev(G, dtype), tA, tB, fa, fb, bias=tb, act=act, drop=drop, gated=gated, want_dbias=True)
    want, tols = lo.dense_bwd(G.astype(np.float64), parts, dtype == "bf16")
    near(dA, want[0], tols[0], dtype)
    near(dB, want[1], tols[1], dtype)
    near(db, want[2], tols[2], "f32")


@pytest.mark.gpu
@pytest.mark.parametrize("M", [1, 2, 15, 16, 17, 33, 48, 63, 64])
def test_few_rows(M):
    for k, (N, K) in enumerate([(1, 1), (16, 128), (17, 127), (40, 129), (130, 1040), (64, 4096), (333, 2051)]):
        for gated in (False, True):
            run(M * 100 + k, M, N, K, gated=gated, act=(M + k) % 4, dtype=("f32", "bf16")[k % 2], p=0.2 * (k % 3 == 0), train=False)
            run(M * 100 + k, M, N, K, M4E3, (E4M3, M4E3, E5M2)[k % 3], gated=gated, act=(M + k) % 4, bias=k % 2 == 0, residual=False, train=False)


@pytest.mark.gpu
@pytest.mark.parametrize("K", [1, 15, 16, 17, 112, 127, 128, 129, 144, 256, 770, 1000])
def test_ends_of_rows_and_steps(K):
    for k, (M, N) in enumerate([(65, 1), (66, 3), (100, 64), (127, 33), (129, 130), (300, 70)]):
        run(K * 10 + k, M, N, K, gated=k % 2 == 1, act=(K + k) % 4, dtype=("f32", "bf16")[(K + k) % 2], p=0.1 * (k % 2))


@pytest.mark.gpu
@pytest.mark.parametrize("fa,fb", [(M4E3, M4E3), (E4M3, M4E3), (M4E3, E4M3), (E5M2, E5M2), (E2M5, E5M2)])
def test_other_formats(fa, fb):
    for k, (M, N, K) in enumerate([(70, 40, 33), (130, 200, 128), (257, 66, 300)]):
        run(k + 900, M, N, K, fa, fb, gated=k == 1, act=k + 1, dtype=("f32", "bf16")[k % 2], p=0.1 * (k == 2))


@pytest.mark.gpu
@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("M,N,K", [(2040, 1601, 48), (4095, 3201, 130), (4096, 3328, 256)])
def test_large_tiles(M, N, K, gated):
    # enough tiles of 128 x 128 and of 256 x 256 to be taken; the last ones end inside
    run(M + N, M, N // 2 if gated else N, K, gated=gated, act=3 if gated else 1, p=0.1, dtype="bf16" if N == 3201 else "f32")


@pytest.mark.gpu
def test_long_sums_in_slices():
    for k, (M, N, K) in enumerate([(70, 64, 9000), (130, 100, 5000), (3000, 66, 130), (66, 3000, 130), (5000, 40, 40)]):
        for gated in (False, True):
            run(k + 50, M, N, K, gated=gated, act=3, dtype=("f32", "bf16")[k % 2])


@pytest.mark.gpu
@pytest.mark.parametrize("fmt", [(4, 3, 8), (3, 4, 5), (5, 2, 14)])
def test_codes_out(fmt):
    for M, N, K in ((5, 50, 200), (150, 131, 300)):
        for gated in (False, True):
            A, B, fa, fb, b, R, _, _, _ = problem(M, M, N, K, E4M3, E4M3, gated, True, "f32", True, 0.0)
            y64, tol, _ = lo.dense(A, B, fa, fb, b.astype(np.float64), 2, gated, None, R.astype(np.float64))
            y = lb.dense(dev(A), dev(B), fa, fb, bias=dev(b), act=lb.ACT_GELU, residual=dev(R), gated=gated, out_dtype=torch.uint8, out_fmt=fmt)
            lo.check_codes(y.cpu().numpy(), y64, tol, fmt)


@pytest.mark.gpu
def test_every_code_of_every_format():
    # A: one row for each code; B: ones; the sums are the codes' values exactly
    for fmt in (E4M3, M4E3, E5M2, E2M5):
        c = np.arange(256, dtype=np.uint8)
        if fmt[0] == 4:
            c = c[(c & 127) != 127]
        one = np.argmin(np.abs(lo.code_values(*fmt) - 1.0))
        assert lo.code_values(*fmt)[one] == 1.0
        for rows in (c, c[:40]):
            A = np.zeros((len(rows), 130), np.uint8)
            A[:, 129] = rows
            y = lb.dense(dev(A), dev(np.full((3, 130), one, np.uint8)), fmt, fmt)
            assert np.array_equal(y.cpu().numpy(), np.repeat(lo.code_values(*fmt)[rows][:, None], 3, 1).astype(np.float32))


@pytest.mark.gpu
def test_exact_sums_and_repeats():
    # small integers: every sum is exact, whatever the order
    rng = np.random.default_rng(3)
    pick = np.array([0x00, 0x38, 0x40, 0x44, 0xB8, 0xC0, 0xC4], np.uint8)             # 0, 1, 2, 3, -1, -2, -3
    for M, N, K in ((30, 70, 500), (700, 260, 1111), (4096, 3328, 640)):
        A, B = pick[rng.integers(0, 7, (M, K))], pick[rng.integers(0, 7, (N, K))]
        a, b = lo.code_values(4, 3, 7)[A], lo.code_values(4, 3, 7)[B]
        G = rng.integers(-8, 9, (M, N)).astype(np.float32)
        y = lb.dense(dev(A), dev(B))
        assert np.array_equal(host(y), a @ b.T)
        for dtype in ("f32", "bf16"):
            out = lb.dense_bwd(dev(G, dtype), dev(A), dev(B), want_dbias=True)
            for got, want in zip(out, (G @ b, G.T @ a, G.sum(0))):
                want = want if got.dtype == torch.float32 else lo.bf16(want)
                assert np.array_equal(host(got), want)
    A, B, fa, fb, b, R, G, drop, _ = problem(7, 517, 390, 1003, E4M3, M4E3, True, True, "f32", True, 0.1)
    args = (dev(A), dev(B), fa, fb)
    first = lb.dense(*args, bias=dev(b), act=3, residual=dev(R), drop=drop, gated=True), lb.dense_bwd(dev(G), *args, bias=dev(b), act=3, drop=drop, gated=True, want_dbias=True)
    for _ in range(3):
        again = lb.dense(*args, bias=dev(b), act=3, residual=dev(R), drop=drop, gated=True), lb.dense_bwd(dev(G), *args, bias=dev(b), act=3, drop=drop, gated=True, want_dbias=True)
        assert torch.equal(first[0], again[0]) and all(torch.equal(x, y) for x, y in zip(first[1], again[1]))


@pytest.mark.gpu
@pytest.mark.parametrize("M,N,K", [(3985, 771, 770), (8192, 304, 2048), (257, 5000, 1300), (70, 1024, 1024), (9000, 2100, 1030), (2048, 2048, 4096)])
def test_exact_gradients_in_every_tile(M, N, K):
    # small integers again, at sizes that take tiles of every shape, whole and in slices
    rng = np.random.default_rng(M)
    pick = np.array([0x00, 0x38, 0x40, 0xB8, 0xC0], np.uint8)                         # 0, 1, 2, -1, -2
    A, B = pick[rng.integers(0, 5, (M, K))], pick[rng.integers(0, 5, (N, K))]
    a, b = (lo.code_values(4, 3, 7)[v].astype(np.float32) for v in (A, B))           # float32 sums of these are exact in any order
    G = rng.integers(-8, 9, (M, N)).astype(np.float32)
    for dtype in ("f32", "bf16"):
        out = lb.dense_bwd(dev(G, dtype), dev(A), dev(B), want_dbias=True)
        for got, want in zip(out, (G @ b, G.T @ a, G.sum(0))):
            want = want if got.dtype == torch.float32 else lo.bf16(want)
            assert np.array_equal(host(got), want)


@pytest.mark.gpu
def test_parts_of_the_gradients():
    A, B, fa, fb, b, _, G, _, _ = problem(8, 200, 90, 75, E4M3, E4M3, False, True, "f32", False, 0.0)
    args = (dev(G), dev(A), dev(B), fa, fb)
    every = lb.dense_bwd(*args, bias=dev(b), act=2, want_dbias=True)
    for k in range(3):
        got = lb.dense_bwd(*args, bias=dev(b), act=2, want_da=k == 0, want_db=k == 1, want_dbias=k == 2)
        assert torch.equal(got[k], every[k]) and all(got[j] is None for j in range(3) if j != k)


@pytest.mark.gpu
def test_differences():
    # along a direction of bias and of the operands' values: the loss sum(G * y)
    rng = np.random.default_rng(5)
    M, N, K, eps = 80, 24, 48, 2.0 ** -6
    for gated in (False, True):
        A, B, fa, fb, b, R, G, drop, f = problem(11, M, N, K, E4M3, E4M3, gated, True, "f32", True, 0.2)
        dA, dB, db = (host(t) for t in lb.dense_bwd(dev(G), dev(A), dev(B), fa, fb, bias=dev(b), act=3, drop=drop, gated=gated, want_dbias=True))
        loss = lambda bias: float((G.astype(np.float64) * host(lb.dense(dev(A), dev(B), fa, fb, bias=dev(bias), act=3, residual=dev(R), drop=drop, gated=gated))).sum())  # noqa: E731
        v = np.sign(rng.standard_normal(b.shape)).astype(np.float32)
        slope = (loss(b + np.float32(eps) * v) - loss(b - np.float32(eps) * v)) / (2 * eps)
        scale = np.sqrt((G.astype(np.float64) ** 2 * (1 if f is None else f ** 2)).sum()) * (4 if gated else 1)
        assert abs(slope - (db * v).sum()) <= 2e-2 * scale, gated
        # one operand's values a code up and down: the sums move by a whole code, so the oracle in 64 bits takes the differences
        a, w = lo.code_values(*fa)[A], lo.code_values(*fb)[B]

        def exact(a, w):
            z = a @ w.T + b
            v = lo.act(z[:, :N] if gated else z, 3)[0] * (z[:, N:] if gated else 1)
            return float((G * v * f).sum())
        va, vw = rng.standard_normal(a.shape), rng.standard_normal(w.shape)
        h = 1e-6
        sa, sw = (exact(a + h * va, w) - exact(a - h * va, w)) / (2 * h), (exact(a, w + h * vw) - exact(a, w - h * vw)) / (2 * h)
        assert abs(sa - (dA * va).sum()) <= 1e-4 * np.linalg.norm(dA) * np.linalg.norm(va)
        assert abs(sw - (dB * vw).sum()) <= 1e-4 * np.linalg.norm(dB) * np.linalg.norm(vw)


@pytest.mark.gpu
def test_views_leading_axes_streams_and_empty():
    rng = np.random.default_rng(6)
    A, B = codes(rng, (2, 50, 100), E4M3), codes(rng, (40, 100), E4M3)
    y = lb.dense(dev(A), dev(B), E4M3, E4M3)
    assert y.shape == (2, 50, 40)
    flat = dev(np.concatenate([np.zeros(3, np.uint8), A.ravel()]))[3:].view(100, 100)     # off every alignment
    assert torch.equal(lb.dense(flat, dev(B), E4M3, E4M3), y.view(100, 40))
    wide = dev(np.concatenate([A.reshape(100, 100), A.reshape(100, 100)], 1))
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    z = lb.dense(wide[:, 100:], dev(B.T.copy()).t(), E4M3, E4M3, stream=s)
    g = lb.dense_bwd(y, dev(A), dev(B), E4M3, E4M3, act=2, stream=s)
    s.synchronize()
    assert torch.equal(z, y.view(100, 40)) and g[0].shape == A.shape and g[1].shape == B.shape
    want = lb.dense_bwd(y, dev(A), dev(B), E4M3, E4M3, act=2)
    assert torch.equal(g[0], want[0]) and torch.equal(g[1], want[1])
    e = torch.empty(0, 100, dtype=torch.uint8, device=DEV)
    assert lb.dense(e, dev(B)).shape == (0, 40)
    dA, dB, db = lb.dense_bwd(torch.empty(0, 40, device=DEV), e, dev(B), want_dbias=True)
    assert dA.shape == (0, 100) and (dB == 0).all() and (db == 0).all()
    k0 = torch.empty(70, 0, dtype=torch.uint8, device=DEV)
    b = torch.randn(9, device=DEV)
    assert torch.equal(lb.dense(k0, torch.empty(9, 0, dtype=torch.uint8, device=DEV), bias=b), b.expand(70, 9))
    _, _, db = lb.dense_bwd(torch.ones(70, 9, device=DEV), k0, torch.empty(9, 0, dtype=torch.uint8, device=DEV), want_dbias=True)
    assert (db == 70).all()


@pytest.mark.gpu
def test_graph_replays():
    rng = np.random.default_rng(9)
    A, B = dev(codes(rng, (200, 131), E4M3)), dev(codes(rng, (60, 131), E4M3))
    G = torch.randn(200, 30, device=DEV)
    step = torch.zeros(1, dtype=torch.int64, device=DEV)
    call = lambda d: (lb.dense(A, B, E4M3, E4M3, act=3, drop=d, gated=True), *lb.dense_bwd(G, A, B, E4M3, E4M3, act=3, drop=d, gated=True, want_dbias=True))  # noqa: E731
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        call((0.3, 1, 10, step))
    torch.cuda.current_stream().wait_stream(s)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        outs = call((0.3, 1, 10, step))
    for k in range(4):
        step.fill_(k)
        A.copy_(dev(codes(rng, (200, 131), E4M3)))
        G.normal_()
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(outs, call((0.3, 1, 10 + k))))


@pytest.mark.gpu
def test_offsets_beyond_32_bits():
    rng = np.random.default_rng(10)
    M, N, K = 131080, 32800, 16
    A, B = codes(rng, (M, K), E4M3), codes(rng, (N, K), E4M3)
    y = lb.dense(dev(A), dev(B), E4M3, E4M3, out_dtype=torch.uint8, out_fmt=(4, 3, 0))
    rows = np.array([0, 65535, 65536, M - 300, M - 1])
    y64, tol, _ = lo.dense(A[rows], B, E4M3, E4M3, None, 0, False, None, None)
    lo.check_codes(y[torch.from_numpy(rows).to(DEV)].cpu().numpy(), y64, tol, (4, 3, 0))
    del y
    M, N = 70000, 65600                                            # the gradient matrix and its transpose
    A, B = codes(rng, (M, K), E4M3), codes(rng, (N, K), E4M3)
    G = torch.randn(M, N, device=DEV, dtype=torch.bfloat16)
    dA, dB, db = lb.dense_bwd(G, dev(A), dev(B), E4M3, E4M3, want_dbias=True)
    a, b = lo.code_values(*E4M3)[A], lo.code_values(*E4M3)[B]
    for rows, got, other, pick in ((np.array([0, 40000, M - 1]), dA, b, lambda r: host(G[r])), (np.array([0, 40000, N - 1]), dB, a, lambda r: host(G[:, r].t()))):
        r = torch.from_numpy(rows).to(DEV)
        g = pick(r)
        near(got[r], g @ other, (g.shape[1] + 16) * lo.U * (np.abs(g) @ np.abs(other)), "bf16")
    g = host(G[:, -1])
    assert abs(host(db)[-1] - g.sum()) <= (M + 64) * lo.U * np.abs(g).sum()


@pytest.mark.gpu
@pytest.mark.parametrize("M,N", [(1 << 27, 32), (1 << 13, 1 << 20)])
def test_many_tiles(M, N):
    # millions of tiles of 64 x 64; small integers
    K = 32
    gen = torch.Generator(device=DEV).manual_seed(M)
    pick = torch.tensor([0x00, 0x38, 0x40, 0xB8, 0xC0], dtype=torch.uint8, device=DEV)       # 0, 1, 2, -1, -2
    value = torch.tensor([0.0, 1.0, 2.0, -1.0, -2.0], device=DEV)
    a, b = (torch.randint(0, 5, (r, K), generator=gen, device=DEV, dtype=torch.uint8) for r in (M, N))
    take = lambda table, i: torch.index_select(table, 0, i.reshape(-1).int()).view(i.shape)  # noqa: E731
    A, B = torch.empty_like(a), take(pick, b)
    step = M // 16
    for m in range(0, M, step):
        A[m:m + step] = take(pick, a[m:m + step])
    y = lb.dense(A, B, out_dtype=torch.bfloat16)
    for m in range(0, M, step):
        w = take(value, a[m:m + step]) @ take(value, b).t().contiguous()
        assert torch.equal(y[m:m + step], w.bfloat16()), m


@pytest.mark.gpu
def test_gradients_of_long_rows():
    # rows of which 64 take more than 2^32 bytes; small integers: every sum is exact
    M, N, K = 64, 8, 17_100_003
    gen = torch.Generator(device=DEV).manual_seed(4)
    pick = torch.tensor([0x00, 0x38, 0x40, 0xB8, 0xC0], dtype=torch.uint8, device=DEV)       # 0, 1, 2, -1, -2
    value = torch.tensor([0.0, 1.0, 2.0, -1.0, -2.0], device=DEV)
    a, b = (torch.randint(0, 5, (r, K), generator=gen, device=DEV, dtype=torch.uint8) for r in (M, N))
    take = lambda table, i: torch.index_select(table, 0, i.reshape(-1).int()).view(i.shape)  # noqa: E731
    A, B = take(pick, a), take(pick, b)
    G = torch.randint(-8, 9, (M, N), generator=gen, device=DEV).float()
    dA, dB, db = lb.dense_bwd(G, A, B, want_dbias=True)
    for k in range(0, K, 1 << 21):
        s = slice(k, min(k + (1 << 21), K))
        assert torch.equal(dA[:, s], G @ take(value, b[:, s])) and torch.equal(dB[:, s], G.t().contiguous() @ take(value, a[:, s])), k
    assert torch.equal(db, G.sum(0))


def test_refusals():
    P, W, f, d = ctypes.c_void_p(0x1000), ctypes.c_void_p(0x2000), (4, 3, 7), lb.lba_drop(0.0, 0, 0, None)
    base = dict(A=P, B=P, M=100, N=8, K=32, fa=f, fb=f, gated=0, bias=None, act=0, drop=d, R=None, rt=0, Y=P, yt=0, yf=f, ws=None, n=0)
    call = lambda **k: lb.lba_dense(*{**base, **k}.values())  # noqa: E731
    assert call(A=None) == lb.ERR_NULL and call(B=None) == lb.ERR_NULL and call(Y=None) == lb.ERR_NULL
    assert call(M=-1) == lb.ERR_SHAPE and call(M=(1 << 30) + 1) == lb.ERR_SHAPE and call(N=(1 << 20) + 1) == lb.ERR_SHAPE and call(K=(1 << 30) + 1) == lb.ERR_SHAPE
    assert call(fa=(6, 1, 7)) == lb.ERR_FORMAT and call(fb=(4, 3, 40)) == lb.ERR_FORMAT and call(yt=2, yf=(4, 4, 7)) == lb.ERR_FORMAT
    assert call(act=9) == lb.ERR_UNSUPPORTED and call(yt=7) == lb.ERR_UNSUPPORTED and call(R=P, rt=2) == lb.ERR_UNSUPPORTED
    assert call(drop=lb.lba_drop(1.1, 0, 0, None)) == lb.ERR_FORMAT
    assert call(M=0) == lb.OK and call(N=0, A=None) == lb.OK
    need = lb.lba_dense_workspace_bytes(100, 8, 33, f, f, 0)
    assert need > 0 and lb.lba_dense_workspace_bytes(4, 8, 33, f, f, 0) == 0 and lb.lba_dense_workspace_bytes(100, 8, 33, (1, 6, 0), f, 0) == 0
    assert call(K=33) == lb.ERR_NULL and call(K=33, ws=W, n=need - 1) == lb.ERR_SHAPE and call(K=33, ws=ctypes.c_void_p(0x2010), n=need) == lb.ERR_ALIGN
    base2 = dict(G=P, gt=0, A=P, B=P, M=100, N=8, K=32, fa=f, fb=f, gated=0, bias=None, act=2, drop=d, dA=P, dB=P, db=P, ws=W, n=1 << 40)
    back = lambda **k: lb.lba_dense_bwd(*{**base2, **k}.values())  # noqa: E731
    assert back(G=None) == lb.ERR_NULL and back(A=None) == lb.ERR_NULL and back(dA=None, dB=None, db=None) == lb.ERR_NULL
    assert back(gt=2) == lb.ERR_UNSUPPORTED and back(act=4) == lb.ERR_UNSUPPORTED and back(N=-1) == lb.ERR_SHAPE
    assert back(ws=None) == lb.ERR_NULL and back(n=100) == lb.ERR_SHAPE and back(ws=ctypes.c_void_p(0x2008)) == lb.ERR_ALIGN
    with pytest.raises(TypeError):
        lb.dense(torch.zeros(2, 3, dtype=torch.uint8), torch.zeros(2, 3, dtype=torch.uint8))

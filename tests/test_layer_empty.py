"""The layer operators on empty batches and rows: an empty tensor's address is null, which asks for nothing and is no error."""
import ctypes

import pytest
import torch

from paper_2401_14110_amd import binding as lb

F = (4, 3, 7)
NO = lb.lba_drop(0.0, 0, 0, None)
P = ctypes.c_void_p(0x1000)


def norm_bwd(M, N, **k):
    return lb.lba_layernorm_bwd(*{**dict(G=None, gt=0, X=None, xt=0, gamma=None, m=None, r=None, dX=None, dg=None, db=None, M=M, N=N, ws=None, n=0), **k}.values())


def drop_bwd(M, N, **k):
    return lb.lba_dropout_bwd(*{**dict(G=None, gt=0, X=None, xt=0, scale=1.0, bias=None, act=0, drop=NO, dX=None, db=None, M=M, N=N, ws=None, n=0), **k}.values())


def dense_bwd(M, N, K, **k):
    return lb.lba_dense_bwd(*{**dict(G=None, gt=0, A=None, B=None, M=M, N=N, K=K, fa=F, fb=F, gated=0, bias=None, act=0, drop=NO, dA=None, dB=None, db=None, ws=None,
                                     n=0), **k}.values())


def test_empty_outputs_are_no_error():
    for call in (norm_bwd, drop_bwd):
        assert call(0, 8) == lb.OK and call(8, 0) == lb.OK and call(0, 0) == lb.OK
        assert call(8, 8) == lb.ERR_NULL and call(-1, 8) == lb.ERR_SHAPE and call(0, 8, gt=7) == lb.ERR_UNSUPPORTED
    assert dense_bwd(0, 8, 8) == lb.OK and dense_bwd(8, 0, 8) == lb.OK and dense_bwd(8, 8, 0) == lb.OK and dense_bwd(0, 0, 0, gated=1) == lb.OK
    assert dense_bwd(8, 8, 8) == lb.ERR_NULL and dense_bwd(0, -1, 8) == lb.ERR_SHAPE and dense_bwd(0, 8, 8, act=5) == lb.ERR_UNSUPPORTED
    assert dense_bwd(8, 8, 0, G=P, fa=(6, 1, 7)) == lb.ERR_FORMAT


@pytest.mark.gpu
def test_calls_on_empty_batches():
    e, z, v = torch.empty(0, 40, device="cuda"), torch.empty(0, device="cuda"), torch.randn(40, device="cuda")
    for params in (False, True):
        dx, dg, db = lb.layernorm_bwd(e, e, v, z, z, want_params=params)
        assert dx.shape == (0, 40) and (not params or not (dg.any() or db.any()))
    assert lb.dropout_bwd(e, (0.1, 1, 2))[0].shape == (0, 40)
    dx, db = lb.dropout_bwd(e, (0.1, 1, 2), x=e, bias=v, act=2, want_dbias=True)
    assert dx.shape == (0, 40) and not db.any()
    rows = torch.empty(0, 3, 100, dtype=torch.uint8, device="cuda")
    B = torch.randint(0, 112, (40, 100), dtype=torch.uint8, device="cuda")
    for da, dw, gated in ((True, False, False), (True, True, False), (False, True, True), (True, False, True)):
        G = torch.empty(0, 3, 20 if gated else 40, device="cuda")
        dA, dB, _ = lb.dense_bwd(G, rows, B, act=2, gated=gated, want_da=da, want_db=dw)
        assert (dA.shape == rows.shape) if da else dA is None
        assert (dB.shape == B.shape and not dB.any()) if dw else dB is None
    # sums over no codes, with and without the bias's gradient
    a0, b0 = torch.empty(70, 0, dtype=torch.uint8, device="cuda"), torch.empty(40, 0, dtype=torch.uint8, device="cuda")
    dA, dB, db = lb.dense_bwd(torch.ones(70, 40, device="cuda"), a0, b0)
    assert dA.shape == (70, 0) and dB.shape == (40, 0) and db is None
    assert (lb.dense_bwd(torch.ones(70, 40, device="cuda"), a0, b0, want_dbias=True)[2] == 70).all()
    # no columns of outputs
    dA, dB, _ = lb.dense_bwd(torch.empty(70, 0, device="cuda"), torch.zeros(70, 100, dtype=torch.uint8, device="cuda"), B[:0])
    assert dA.shape == (70, 100) and not dA.any() and dB.shape == (0, 100)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_statistics_of_rows_of_nothing(dtype):
    x, v = torch.empty(300, 0, device="cuda", dtype=dtype), torch.empty(0, device="cuda")
    junk = [torch.zeros(300, device="cuda") for _ in range(4)]       # memory that the statistics are likely to be given
    del junk
    for kw in (dict(), dict(gamma=v, beta=v), dict(out_dtype=torch.uint8, out_fmt=F)):
        y, mean, rstd = lb.layernorm(x, want_stats=True, **kw)
        assert y.shape == (300, 0) and mean.shape == rstd.shape == (300,)
        assert mean.isnan().all() and rstd.isnan().all()             # 0 / 0
    assert lb.layernorm(x).shape == (300, 0)
    dx, dg, db = lb.layernorm_bwd(x, x, None, mean, rstd)
    assert dx.shape == (300, 0) and dg.shape == db.shape == (0,)

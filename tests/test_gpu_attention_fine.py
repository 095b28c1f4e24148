"""What bfloat16 inputs may ask for: weights that are not rounded to bfloat16 for any output type of both attentions, whose bounds are those of float32, and
gradients without the rounding of O for any query."""
import ctypes

import numpy as np
import pytest
import torch

import attention_oracle as ao
import layer_oracle as lo
from paper_2401_14110_amd import binding as lb
from test_gpu_attention import desc, starts
from test_gpu_attention_offset import against_the_formulas
from test_gpu_cache import a_table, expected, filled, ints, on_device
from test_gpu_layernorm import DEV, dev, near, values

FORMATS = [(4, 3, 7 + 6), (3, 4, 3 + 2), (5, 2, 15)]


@pytest.mark.gpu
@pytest.mark.parametrize("lens,H,KV,D,causal", [([1], 1, 1, 1, True), ([33, 0, 130], 4, 2, 64, True), ([200, 65], 6, 2, 83, False), ([300], 2, 1, 128, True), ([2, 129], 3, 3, 96, True),
                                               ([1, 1500], 1, 1, 32, False)])
def test_packed_sequences(lens, H, KV, D, causal):
    rng = np.random.default_rng(sum(lens))
    x = [values(rng, (sum(lens), h, D), "bf16") for h in (H, KV, KV)]
    want, tol = ao.packed(*x, lens, lens, causal, float(np.float32(D ** -0.5)), "f32")["o"]
    q, k, v = (dev(t, "bf16") for t in x)
    kw = dict(starts=starts(lens), causal=causal, fine=True)
    got, lse = lb.attention(q, k, v, want_stats=True, **kw)
    assert got.dtype == torch.bfloat16 and got.isfinite().all()
    near(got, want, tol, "bf16")
    assert torch.equal(lse, lb.attention(q, k, v, want_stats=True, **{**kw, "fine": False})[1])
    whole = lb.attention(q, k, v, out_dtype=torch.float32, **kw)
    assert torch.equal(whole, lb.attention(q, k, v, out_dtype=torch.float32, **{**kw, "fine": False}))
    assert torch.equal(got, whole.bfloat16())            # one rounding of the same sums
    for fmt in FORMATS:
        codes = lb.attention(q, k, v, out_dtype=torch.uint8, out_fmt=fmt, **kw)
        lo.check_codes(codes.cpu().numpy(), want, tol + 2 * lo.U * np.abs(want), fmt)
        assert torch.equal(codes, lb.dropout(whole, None, out_dtype=torch.uint8, out_fmt=fmt))
    f = [t.float() for t in (q, k, v)]                   # float32 has whole weights in any case
    assert torch.equal(lb.attention(*f, **kw), lb.attention(*f, **{**kw, "fine": False}))


@pytest.mark.gpu
@pytest.mark.parametrize("lens,fresh,H,KV,D,page", [([1], 1, 1, 1, 32, 1), ([129, 40], 1, 12, 12, 64, 16), ([700, 3, 0], 2, 8, 2, 128, 64), ([5000], 1, 6, 1, 96, 7), ([90, 17], 33, 2, 1, 64, 16)])
def test_over_the_cache(lens, fresh, H, KV, D, page):
    rng = np.random.default_rng(sum(lens))
    table, pages = a_table(rng, len(lens), -(-max(lens) // page))
    arrays = filled(rng, pages, KV, page, D)
    x = values(rng, (len(lens), fresh, H, D), "bf16")
    want, tol = expected(arrays, table, x, lens, page, "f32", D ** -0.5)
    q, cache, t, n = dev(x, "bf16"), on_device(arrays), torch.from_numpy(table).to(DEV), ints(lens)
    got = lb.cache_attention(q, cache, t, n, fine=True)
    assert got.dtype == torch.bfloat16 and got.isfinite().all()
    near(got, want, tol, "bf16")
    whole = lb.cache_attention(q, cache, t, n, out_dtype=torch.float32)
    assert torch.equal(got, whole.bfloat16()) and torch.equal(whole, lb.cache_attention(q, cache, t, n, out_dtype=torch.float32, fine=True))
    for fmt in FORMATS:
        codes = lb.cache_attention(q, cache, t, n, out_dtype=torch.uint8, out_fmt=fmt, fine=True)
        lo.check_codes(codes.cpu().numpy(), want, tol + 2 * lo.U * np.abs(want), fmt)


@pytest.mark.gpu
@pytest.mark.parametrize("mean", [0.0, 1.0, 64.0])
@pytest.mark.parametrize("lens,lens_k,H,KV,D,causal", [([700, 3, 0, 513], [700, 3, 0, 513], 2, 1, 64, True), ([40, 600], [1100, 577], 1, 1, 83, False), ([1500], [1500], 1, 1, 128, True),
                                                       ([1500], [1500], 1, 1, 128, False), ([2, 200], [2, 200], 2, 2, 32, True)])
def test_gradients_of_all_queries(lens, lens_k, H, KV, D, causal, mean):
    against_the_formulas(lens, lens_k, H, KV, D, causal, mean, True)


@pytest.mark.gpu
def test_gradients_in_float32_and_workspaces():
    q = torch.randn(300, 2, 40, device="cuda")
    o, lse = lb.attention(q, q, q, want_stats=True)
    for a, b in zip(lb.attention_bwd(q, q, q, q, o, lse), lb.attention_bwd(q, q, q, q, o, lse, fine=True)):
        assert torch.equal(a, b)


def test_refusals():
    P, f = ctypes.c_void_p(0x1000), (4, 3, 7)
    for t in (lb.F32, lb.BF16):                          # the same workspaces
        for name in (lb.lba_attention_workspace_bytes, lb.lba_attention_bwd_workspace_bytes):
            for k in (dict(T=8, Tk=8), dict(T=128, Tk=4096)):
                assert name(desc(type=t, **k)) == name(desc(type=t | lb.FINE, **k))
    s = lb.lba_strides(64, 16)
    back = lambda t: lb.lba_attention_bwd(desc(type=t, T=0, Tk=0), P, P, P, P, P, P, P, s, P, s, P, s, P, 1 << 20)  # noqa: E731
    call = lambda t, o=0, **k: lb.lba_attention(desc(type=t, **k), P, P, P, P, o, f, None, None, 0)  # noqa: E731
    over = lambda t, fresh=1: lb.lba_cache_attention(lb.lba_cache4(P, P, P, P, 4, 2, 2, P, P, 16, 2, 64), P, lb.lba_strides(128, 64), t, fresh, 4, 0.1, P, 0, f, P, 1 << 20)  # noqa: E731
    for fn in (call, back, over):
        assert fn(lb.FINE | 2) == lb.ERR_UNSUPPORTED and fn(2 * lb.FINE) == lb.ERR_UNSUPPORTED
    assert call(lb.FINE | lb.BF16, T=0, Tk=0) == lb.OK and back(lb.FINE | lb.BF16) == lb.OK and over(lb.FINE | lb.BF16, 0) == lb.OK
    assert call(lb.BF16, lb.FINE, T=0, Tk=0) == lb.ERR_UNSUPPORTED                   # (of the inputs' type)

"""Weights that are not rounded to bfloat16, on request, for every output type of both attentions: the bounds are those of float32."""
import ctypes

import numpy as np
import pytest
import torch

import attention_oracle as ao
import layer_oracle as lo
from paper_2401_14110_amd import binding as lb
from test_gpu_attention import desc, starts
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


def test_refusals():
    P, f = ctypes.c_void_p(0x1000), (4, 3, 7)
    call = lambda t, **k: lb.lba_attention(desc(**k), P, P, P, P, t, f, None, None, 0)  # noqa: E731
    assert call(lb.FINE | 3) == lb.ERR_UNSUPPORTED and call(2 * lb.FINE) == lb.ERR_UNSUPPORTED and call(lb.FINE | lb.CODE8, T=0, Tk=0) == lb.OK
    cache = lb.lba_cache4(P, P, P, P, 4, 2, 2, P, P, 16, 2, 64)
    over = lambda t, fresh=1: lb.lba_cache_attention(cache, P, lb.lba_strides(128, 64), 0, fresh, 4, 0.1, P, t, f, P, 1 << 20)  # noqa: E731
    assert over(lb.FINE | 3) == lb.ERR_UNSUPPORTED and over(2 * lb.FINE) == lb.ERR_UNSUPPORTED and over(lb.FINE | lb.BF16, 0) == lb.OK

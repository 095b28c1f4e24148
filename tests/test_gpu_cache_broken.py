"""Attention over the cache where some of a call's new tokens see blocks that stand for NaN, or codes beyond the numbers, and others do not: who does not has the bits
that zeros give, who does has them in the blocks' own columns; and a call with many takes about as long as any."""
import time

import numpy as np
import pytest
import torch

from paper_2401_14110_amd import binding as lb
from test_gpu_cache import a_table, filled, ints, on_device

DT = [torch.float32, torch.bfloat16]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", DT)
@pytest.mark.parametrize("what", ["nan", "beyond"])
@pytest.mark.parametrize("lens,fresh,H,KV,D,page", [([40], 3, 4, 2, 64, 16), ([33, 5, 70], 2, 2, 2, 32, 8), ([600, 31], 5, 16, 2, 128, 64), ([3000], 2, 3, 1, 96, 7), ([90, 64], 33, 2, 1, 128, 16),
                                                    ([50], 1, 2, 1, 64, 16)])
def test_blocks_that_some_see(lens, fresh, H, KV, D, page, what, dtype):
    rng = np.random.default_rng(sum(lens))
    table, pages = a_table(rng, len(lens), -(-max(lens) // page))
    arrays = filled(rng, pages, KV, page, D)
    q = torch.randn(len(lens), fresh, H, D, device="cuda", generator=torch.Generator(device="cuda").manual_seed(1)).to(dtype)
    t, ln = torch.from_numpy(table).cuda(), ints(lens)
    # of each sequence a block at the newest token, one a few before, and an old one
    spots = []
    for b, n in enumerate(lens):
        for back in sorted({0, min(fresh // 2, n - 1), min(fresh + 9, n - 1)}):
            p, kv, block = n - 1 - back, int(rng.integers(KV)), int(rng.integers(D // 32))
            spots.append((b, p, kv, block))
            at = (table[b, p // page], kv, p % page)
            if what == "nan":
                arrays[3][at + (block,)] = 255
            else:                                        # the first element 6 * 2^127, another minus that, the others zero
                arrays[3][at + (block,)] = 254
                codes = arrays[2][at]
                codes[16 * block:16 * block + 16] = 0
                codes[16 * block], codes[16 * block + 5] = 7, 15
    zero = [a.copy() for a in arrays]
    for b, p, kv, block in spots:
        zero[3][table[b, p // page], kv, p % page, block] = 0
    cache, clean = on_device(arrays), on_device(zero)
    for kw in (dict(), dict(out_dtype=torch.float32), dict(fine=True)):
        got, want = (lb.cache_attention(q, c, t, ln, **kw) for c in (cache, clean))
        assert want.isfinite().all()
        expect = want.clone()
        for b, p, kv, block in spots:
            first = max(0, p - (lens[b] - fresh))        # the first new token that sees it
            x = expect[b, first:, kv * (H // KV):(kv + 1) * (H // KV), 32 * block:32 * block + 32]
            if what == "nan":
                x.fill_(float("nan"))
            else:
                x[..., 0], x[..., 10] = float("inf"), float("-inf")
        assert torch.equal(got.isnan(), expect.isnan()) and torch.equal(got.nan_to_num(7.0, 9.0, 11.0), expect.nan_to_num(7.0, 9.0, 11.0)), kw


@pytest.mark.gpu
def test_a_batch_with_one_that_has_diverged():
    lens, page, KV, D = [8000] * 8, 64, 8, 128
    table = torch.arange(1000, dtype=torch.int32, device="cuda").view(8, 125)
    cache = lb.kv_cache(1000, page, KV, D)
    for c in cache[::2]:
        c.random_(0, 256)
    q = torch.randn(8, 5, 32, D, device="cuda").bfloat16()
    wide = torch.full((8, 2048), -1, dtype=torch.int32, device="cuda")
    wide[:, :125] = table

    def run(scale):
        cache.k_scale.fill_(127)
        cache.v_scale.fill_(127)
        cache.v_scale[875:] = scale
        lb.cache_attention(q, cache, wide, ints(lens))
        torch.cuda.synchronize()
        begin = time.monotonic()
        for _ in range(10):
            y = lb.cache_attention(q, cache, wide, ints(lens))
        torch.cuda.synchronize()
        return time.monotonic() - begin, y

    broken, y = run(255)
    clean, z = run(127)
    assert y[7].isnan().all() and torch.equal(y[:7], z[:7]) and broken < 10 * clean + 0.01

"""Attention over the cache of float32 queries at the end of the type's range: beyond bfloat16's largest number, 2^128 - 2^120, whose nearest bfloat16 is infinity."""
import numpy as np
import pytest
import torch

from paper_2401_14110_amd import binding as lb
from test_gpu_cache import expected, filled, ints, on_device
from test_gpu_layernorm import DEV, dev, near


@pytest.mark.gpu
@pytest.mark.parametrize("length,fresh,D", [(40, 1, 64), (70, 3, 32), (1500, 2, 128)])
def test_queries_at_the_end_of_the_range(length, fresh, D):
    rng = np.random.default_rng(length)
    page = 16
    pages = -(-length // page)
    arrays = list(filled(rng, pages, 2, page, D))
    arrays[1] = (arrays[1] - 13).astype(np.uint8)        # keys of about 2^-13: D products stay below 2^128
    table = rng.permutation(pages).astype(np.int32)[None]
    top = np.finfo(np.float32).max
    q = rng.standard_normal((1, fresh, 4, D)).astype(np.float32) * np.float32(2.0 ** 120)
    q[:, :, :, 3], q[:, :, 1::2, 7] = top, -np.float32(2.0 ** 128 - 2.0 ** 119)
    scale = 2.0 ** -114
    want, tol = expected(arrays, table, q, [length], page, "f32", scale)
    got = lb.cache_attention(dev(q), on_device(arrays), torch.from_numpy(table).to(DEV), ints([length]), scale=scale)
    assert got.isfinite().all()                          # (which `near` does not say)
    near(got, want, tol, "f32")

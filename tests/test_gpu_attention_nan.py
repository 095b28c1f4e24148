"""A query that holds a NaN has NaN as its output, and nothing else has, however the keys that it sees are cut into parts that are joined."""
import pytest
import torch

from paper_2401_14110_amd import binding as lb

DT = [torch.float32, torch.bfloat16]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", DT)
@pytest.mark.parametrize("length,fresh", [(100, 1), (1500, 1), (1500, 3), (9000, 1), (9000, 2), (70000, 1)])    # one chunk of positions, some, many
def test_over_the_cache(length, fresh, dtype):
    g = torch.Generator(device="cuda").manual_seed(length)
    pages = length // 64 + 1
    cache, table = lb.kv_cache(pages, 64, 2, 64), torch.randperm(pages, device="cuda", generator=g, dtype=torch.int32)[None]
    lens = torch.tensor([length], dtype=torch.int32, device="cuda")
    k, v = (torch.randn(1, length, 2, 64, device="cuda", generator=g) for _ in range(2))
    lb.cache_write(k, v, cache, table, None, lens)
    q = torch.randn(1, fresh, 4, 64, device="cuda", generator=g).to(dtype)
    want = lb.cache_attention(q, cache, table, lens)
    bad = q.clone()
    bad[0, -1, 2, 5] = float("nan")
    for out in (dtype, torch.float32):
        want = lb.cache_attention(q, cache, table, lens, out_dtype=out)
        got = lb.cache_attention(bad, cache, table, lens, out_dtype=out)
        assert got[0, -1, 2].isnan().all()
        got[0, -1, 2] = want[0, -1, 2]
        assert torch.equal(got, want) and want.isfinite().all()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", DT)
@pytest.mark.parametrize("n,m", [(1, 40), (3, 5000), (130, 3000)])
def test_over_keys(n, m, dtype):
    g = torch.Generator(device="cuda").manual_seed(m)
    k, v = (torch.randn(m, 1, 64, device="cuda", generator=g).to(dtype) for _ in range(2))
    q = torch.randn(n, 2, 64, device="cuda", generator=g).to(dtype)
    s, sk = (torch.tensor([0, x], dtype=torch.int32, device="cuda") for x in (n, m))
    want, stats = lb.attention(q, k, v, starts=s, starts_k=sk, want_stats=True)
    bad = q.clone()
    bad[-1, 1, 5] = float("nan")
    got, lse = lb.attention(bad, k, v, starts=s, starts_k=sk, want_stats=True)
    assert got[-1, 1].isnan().all() and lse[-1, 1].isnan()
    got[-1, 1], lse[-1, 1] = want[-1, 1], stats[-1, 1]
    assert torch.equal(got, want) and torch.equal(lse, stats) and want.isfinite().all()

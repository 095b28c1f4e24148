"""What the attention calls copy (a list of starts that is a column, heads whose elements are not neighbours) lives until the kernels are launched: the
library gets addresses only, and a block freed before is the next output's or workspace's."""
import weakref

import numpy as np
import pytest
import torch

from paper_2401_14110_amd import binding as lb


class OnDevice(torch.Tensor):
    """Host memory that passes for a device's."""

    def get_device(self):
        return 0


class Library:
    """Takes every call and looks, when it comes, whether the copies are still there."""

    def __init__(self, copies):
        self.copies, self.calls = copies, []

    def __getattr__(self, name):
        if name.endswith("_bytes"):
            return lambda *a: 512
        return lambda *a: (self.calls.append((name, [c() is not None for c in self.copies])), lb.OK)[1]


@pytest.fixture
def library(monkeypatch):
    copies, real = [], lb._whole

    def whole(t, on):
        got = real(t, on)
        if got is not t:
            copies.append(weakref.ref(got))
        return got

    got = Library(copies)
    monkeypatch.setattr(lb, "_whole", whole)
    monkeypatch.setattr(lb, "lib", lambda: got)
    monkeypatch.setattr(lb, "_on", lambda stream, device: (None, None))
    monkeypatch.setattr(lb, "_attn_bytes_of", lambda *a: 512)
    return got


def strided(t):
    """The same with no two elements neighbours."""
    return torch.stack([t, t], -1)[..., 0].as_subclass(OnDevice)


def ints(*v):
    return torch.tensor(v, dtype=torch.int32)


def test_copies_live_until_the_launch(library):
    x = strided(torch.zeros(8, 2, 32))
    s, sk, lens, table, positions = (strided(t) for t in (ints(0, 3, 8), ints(0, 3, 8), ints(3, 5), ints(0, 1).view(2, 1), torch.arange(8)))
    freq = strided(torch.ones(4, dtype=torch.float64))
    o, lse = x, strided(torch.zeros(8, 2))
    cache = lb.KVCache(*(t.as_subclass(OnDevice) for t in lb.kv_cache(2, 8, 2, 32, device="cpu")))
    whole = torch.zeros(8, 2, 32).as_subclass(OnDevice)
    for call, copies in ((lambda: lb.attention(x, x, x, starts=s, want_stats=True), 4), (lambda: lb.attention(x, x, x, starts=s, starts_k=sk), 5),
                         (lambda: lb.attention(whole, whole, whole, starts=s), 1), (lambda: lb.attention_bwd(whole, whole, whole, whole, whole, lse, starts=s, starts_k=sk), 3),
                         (lambda: lb.attention_bwd(x, x, x, x, o, lse, starts=s), 7), (lambda: lb.rope(x, positions, freq), 3), (lambda: lb.rope_bwd(x, positions, freq), 3),
                         (lambda: lb.cache_write(x, x, cache, table, s, lens), 5), (lambda: lb.cache_read(cache, table, s, lens, 8), 3),
                         (lambda: lb.cache_attention(x[:2], cache, table, lens), 3)):
        del library.copies[:], library.calls[:]
        call()
        (name, alive), = library.calls
        assert len(alive) == copies and all(alive), (name, alive)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("lens", [[3, 5], [1, 0, 2], [40, 90, 7], [300, 0, 500]])
def test_lists_that_are_columns(lens, dtype):
    """Outputs, statistics and workspaces of a few rows, of the size of the list's own block, and larger ones."""
    g = torch.Generator(device="cuda").manual_seed(len(lens))
    T = sum(lens)
    q, G = (torch.randn(T, 4, 64, device="cuda", generator=g).to(dtype) for _ in range(2))
    k, v = (torch.randn(T, 2, 64, device="cuda", generator=g).to(dtype) for _ in range(2))
    s = torch.tensor(np.cumsum([0] + lens), dtype=torch.int32, device="cuda")
    column, other = torch.stack([s, s + 1, -s], 1)[:, 0], torch.stack([s, s], 1).flatten()[::2]
    assert not column.is_contiguous() and not other.is_contiguous()
    for lists, views in ((dict(starts=s), dict(starts=column)), (dict(starts=s, starts_k=s), dict(starts=column, starts_k=other)), (dict(starts=s, starts_k=s), dict(starts=s, starts_k=other))):
        o, lse = lb.attention(q, k, v, want_stats=True, **lists)
        grads = lb.attention_bwd(G, q, k, v, o, lse, **lists)
        for _ in range(3):
            got, stats = lb.attention(q, k, v, want_stats=True, **views)
            assert torch.equal(got, o) and torch.equal(stats, lse)
            assert all(torch.equal(a, b) for a, b in zip(lb.attention_bwd(G, q, k, v, got, stats, **views), grads))

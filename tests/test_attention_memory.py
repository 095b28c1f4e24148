"""Whose pool the outputs and workspaces of the attention calls come from: as in test_layer_memory.py, a call on another stream than the current one takes
nothing from the current one's pool."""
import pytest
import torch

from paper_2401_14110_amd import binding as lb


@pytest.mark.gpu
def test_no_block_of_the_current_stream_is_handed_out(monkeypatch):
    x = torch.randn(700, 3, 2, 40, device="cuda")
    q, k, v = x.unbind(1)
    far = q.transpose(1, 2).contiguous().transpose(1, 2)                             # (D is not along memory: a copy is made)
    starts = torch.tensor([0, 300, 690], dtype=torch.int32, device="cuda")
    positions, freq = torch.arange(700, device="cuda"), torch.rand(8, dtype=torch.float64, device="cuda")
    cache, table = lb.kv_cache(50, 16, 2, 64), torch.arange(50, dtype=torch.int32, device="cuda").view(1, 50)
    lens, keys = torch.tensor([700], dtype=torch.int32, device="cuda"), torch.randn(700, 2, 64, device="cuda")
    lb.cache_write(keys, keys, cache, table, None, lens)
    o, lse = lb.attention(q, k, v, starts=starts, want_stats=True)
    scratch, real = [], lb._scratch

    def spy(*a):
        scratch.append(real(*a))
        return scratch[-1]

    monkeypatch.setattr(lb, "_scratch", spy)
    calls = [lambda s: lb.rope(far, positions, freq, stream=s), lambda s: lb.rope_bwd(q, positions, freq, stream=s),
             lambda s: lb.attention(far, k, v, starts=starts, want_stats=True, stream=s),
             lambda s: lb.attention_bwd(far, q, k, v, o, lse, starts=starts, stream=s),
             lambda s: lb.cache_read(cache, table, None, lens, 700, stream=s),
             lambda s: lb.cache_attention(keys[:1], cache, table, lens, stream=s)]
    side = torch.cuda.Stream()
    torch.cuda.synchronize()

    def memory(call, stream):
        del scratch[:]
        out = call(stream)
        n = 1 if torch.is_tensor(out) else len(out)
        out = [t for t in ((out,) if torch.is_tensor(out) else tuple(out)) + tuple(scratch) if t is not None]
        torch.cuda.synchronize()
        return [(t.data_ptr(), t.data_ptr() + t.numel() * t.element_size()) for t in out], [t.clone() for t in out[:n]]

    workspaces = 0
    for call in calls:
        first, want = memory(call, None)
        second, got = memory(call, side)
        workspaces += sum(t is not None for t in scratch)
        assert all(b <= c or d <= a for a, b in first for c, d in second), call
        assert all(torch.equal(a, b) for a, b in zip(want, got))
    assert workspaces >= 3                               # every call that may need one did

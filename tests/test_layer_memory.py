"""Whose pool the outputs and workspaces of the layer operators come from.  A call on another stream than the current one takes nothing from
the current one's pool: a block that was just freed there may still be read and written by kernels that the call's stream does not wait for."""
import contextlib

import pytest
import torch

from paper_2401_14110_amd import binding as lb


class Stub:
    """A tensor whose memory is known by the stream it was allocated on."""
    shape, device, dtype = (3, 4), "dev", torch.float32

    def __init__(self, pool):
        self.pool, self.recorded = pool, []

    def record_stream(self, stream):
        self.recorded.append(stream)


@pytest.fixture
def pools(monkeypatch):
    now = ["current"]

    @contextlib.contextmanager
    def stream(on):
        now.append(on)
        yield
        now.pop()

    monkeypatch.setattr(torch, "empty", lambda *a, **k: Stub(now[-1]))
    monkeypatch.setattr(torch, "empty_like", lambda *a, **k: Stub(now[-1]))
    monkeypatch.setattr(torch.cuda, "stream", stream)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: now[-1])
    return now


def test_memory_comes_from_the_calls_stream(pools):
    for t in (lb._empty((3, 4), torch.float32, "dev", "side"), lb._empty_as(Stub("current"), torch.uint8, "side")):
        assert t.pool == "side" and t.recorded == ["current"]      # the caller may free it while the current stream reads it
    assert lb._scratch(16, "dev", "side").pool == "side"
    for t in (lb._empty((3, 4), torch.float32, "dev", None), lb._empty_as(Stub("current"), torch.uint8, None), lb._scratch(16, "dev", None)):
        assert t.pool == "current" and t.recorded == []
    assert lb._scratch(0, "dev", None) is None and lb._scratch(0, "dev", "side") is None


@pytest.mark.gpu
def test_no_block_of_the_current_stream_is_handed_out(monkeypatch):
    """Each call on the current stream, its outputs freed, then on another stream: none of the first call's memory comes back."""
    M, N, K = 700, 390, 515
    x, G, v = torch.randn(M, N, device="cuda"), torch.randn(M, N, device="cuda"), torch.randn(N, device="cuda")
    A = torch.randint(0, 112, (M, K), dtype=torch.uint8, device="cuda")
    B = torch.randint(0, 112, (N, K), dtype=torch.uint8, device="cuda")
    _, mean, rstd = lb.layernorm(x, want_stats=True)
    drop, scratch, real = (0.1, 1, 2), [], lb._scratch

    def spy(*a):
        scratch.append(real(*a))
        return scratch[-1]

    monkeypatch.setattr(lb, "_scratch", spy)
    calls = [lambda s: lb.layernorm(x, v, v, want_stats=True, stream=s), lambda s: lb.layernorm_bwd(G, x, v, mean, rstd, stream=s),
             lambda s: lb.dropout(x, drop, bias=v, stream=s), lambda s: lb.dropout_bwd(G, drop, want_dbias=True, stream=s),
             lambda s: lb.dense(A, B, bias=v, stream=s), lambda s: lb.dense_bwd(G, A, B, bias=v, act=2, want_dbias=True, stream=s)]
    side = torch.cuda.Stream()
    torch.cuda.synchronize()

    def memory(call, stream):
        del scratch[:]
        out = call(stream)
        out = [t for t in ((out,) if torch.is_tensor(out) else out) + tuple(scratch) if t is not None]
        torch.cuda.synchronize()
        return [(t.data_ptr(), t.data_ptr() + t.numel() * t.element_size()) for t in out], [t.clone() for t in out[:len(out) - len(scratch)]]

    for call in calls:
        first, want = memory(call, None)
        second, got = memory(call, side)
        assert all(b <= c or d <= a for a, b in first for c, d in second), call
        assert all(torch.equal(a, b) for a, b in zip(want, got))

"""lse, which attention makes itself in every case: rows of no sequence are -infinity, also where the output is given and keeps its own rows there."""
import pytest
import torch

from paper_2401_14110_amd import binding as lb
from test_attention_copies import OnDevice, ints


def test_rows_of_no_sequence_are_set_before_the_launch(monkeypatch):
    """A library that writes nothing leaves what the call has put there, and what memory held before is none of it."""
    class Library:
        def lba_attention(self, *a):
            return lb.OK

    monkeypatch.setattr(lb, "lib", Library)
    monkeypatch.setattr(lb, "_on", lambda stream, device: (None, None))
    monkeypatch.setattr(lb, "_attn_bytes_of", lambda *a: 0)
    monkeypatch.setattr(lb, "_empty", lambda shape, dtype, device, on: torch.full(shape, 7, dtype=dtype))
    q, s = torch.zeros(9, 2, 16).as_subclass(OnDevice), ints(2, 5).as_subclass(OnDevice)
    _, lse = lb.attention(q, q, q, starts=s, out=torch.zeros(9, 2, 16).as_subclass(OnDevice), want_stats=True)
    assert lse.shape == (9, 2) and (lse == -float("inf")).all()


@pytest.mark.gpu
@pytest.mark.parametrize("side", [False, True])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_given_outputs(dtype, side):
    T, H, D, first, lens = 300, 3, 64, 11, [70, 0, 65]
    x = torch.randn(T, H, D, device="cuda").to(dtype)
    s = torch.tensor([first, first + 70, first + 70, first + 135], dtype=torch.int32, device="cuda")
    o, want = lb.attention(x, x, x, starts=s, want_stats=True)
    stream = torch.cuda.Stream() if side else None
    for _ in range(3):
        old = torch.full((T, H), 7.0, device="cuda")     # the block that the statistics may get
        given = torch.full_like(o, 7.0)
        torch.cuda.synchronize()
        del old
        got, lse = lb.attention(x, x, x, starts=s, out=given, want_stats=True, stream=stream)
        torch.cuda.synchronize()
        assert got is given and torch.equal(lse, want) and torch.equal(got[first:first + sum(lens)], o[first:first + sum(lens)])
        assert (got[:first] == 7).all() and (got[first + sum(lens):] == 7).all()
        assert (lse[:first] == -float("inf")).all() and (lse[first + sum(lens):] == -float("inf")).all()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        got, lse = lb.attention(x, x, x, starts=s, out=given, want_stats=True)
    for lens in ([135, 0, 0], [1, 2, 3], [70, 0, 65]):   # replays with other lists: what was a row of a sequence may be none now
        s.copy_(torch.tensor([first, first + lens[0], first + sum(lens[:2]), first + sum(lens)]))
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(lse, lb.attention(x, x, x, starts=s, want_stats=True)[1])

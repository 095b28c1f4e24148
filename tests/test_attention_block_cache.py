"""Prompts of the attention block into a cache: rows that are not the whole of their sequence say so, nothing waits for the host, and a step can be captured."""
import pytest
import torch

from paper_2401_14110_amd import attention as at
from paper_2401_14110_amd import binding as lb


def ints(*v, device="cuda"):
    return torch.tensor(v, dtype=torch.int32, device=device)


def test_one_sequence_takes_no_list_from_the_host(monkeypatch):
    written = []
    block = object.__new__(at.SelfAttention)
    block.heads, block.kv_heads, block.dim, block.causal, block.t_u = 2, 1, 32, True, 6
    block.project = lambda x, positions, train: (None, None, None, torch.zeros(len(x), 4, 32))
    block.finish = lambda u, x, drop=None: x.clone()
    monkeypatch.setattr(lb, "cache_write", lambda *a: written.append(a))
    monkeypatch.setattr(lb, "attention", lambda q, k, v, **kw: q)
    x, lens = torch.zeros(5, 8), ints(5, device="cpu")

    def no_list(*a, **k):
        raise AssertionError("a tensor from host data")

    with monkeypatch.context() as m:
        for name in ("tensor", "as_tensor", "from_numpy"):
            m.setattr(torch, name, no_list)
        y = block.forward(x, torch.arange(5), cache=("held", "table", lens))
    (k, v, held, table, starts, got), = written
    # (as a batch of one: [rows, heads, D] could be a row of each sequence)
    assert k.shape == v.shape == (1, 5, 1, 32) and (held, table, starts, got) == ("held", "table", None, lens)
    assert torch.equal(y, x)
    assert block.forward(x, torch.arange(5), cache=("held", "table", ints(6, device="cpu"))).isnan().all()


@pytest.mark.parametrize("args", [["--rows", "2"], ["--width", "96", "--heads", "4"], ["--width", "512", "--heads", "2"]])
def test_the_command_refuses_what_it_cannot_serve(args, capsys):
    with pytest.raises(SystemExit):
        at.main(["--steps", "1"] + args)
    assert "must be" in capsys.readouterr().err


@pytest.fixture
def server():
    torch.manual_seed(3)
    block = at.SelfAttention(64, 4, 2, 32, seed=2)
    table = ints(8, 1, 6, 3, 0, 7, 2, 5).view(2, 4)
    return block, lambda: lb.kv_cache(9, 8, 2, 32), table


@pytest.mark.gpu
def test_rows_behind_older_tokens(server):
    """The block sees its rows alone, which is not attention over what the sequence holds: NaN there, the cache written all the same."""
    block, cache, table = server
    x, positions = torch.randn(20, 64, device="cuda"), torch.arange(20, device="cuda")
    s, held = ints(2, 9, 9 + 6), cache()                 # two rows before and five behind are of no sequence
    whole = block.forward(x, positions, s, cache=(held, table, ints(7, 6)))
    assert torch.equal(whole, block.forward(x, positions, s)) and whole.isfinite().all()
    for lens, bad in (((12, 6), slice(2, 9)), ((7, 7), slice(9, 15)), ((3, 6), slice(0, 0))):       # (3 of 7 rows are kept: no older ones)
        y = block.forward(x, positions, s, cache=(held, table, ints(*lens)))
        assert y[bad].isnan().all()
        y[bad] = whole[bad]
        assert torch.equal(y, whole)
    # an empty sequence that holds older tokens has no rows here
    y = block.forward(x, positions, ints(2, 9, 9), cache=(held, table, ints(7, 30)))
    assert torch.equal(y[2:9], whole[2:9]) and y.isfinite().all()
    # one sequence, no list
    y = block.forward(x, positions, cache=(held, table[:1], ints(20)))
    assert torch.equal(y, block.forward(x, positions)) and y.isfinite().all()
    assert block.forward(x, positions, cache=(held, table[:1], ints(21))).isnan().all()
    k, _ = lb.cache_read(held, table[:1], None, ints(21), 21, out_dtype=torch.float32)
    assert k[1:].any(-1).all()                           # its rows are the newest
    # and trains so as well
    y, _ = block.forward(x, positions, train=True, cache=(held, table[:1], ints(21)))
    assert y.isnan().all()
    with pytest.raises(ValueError):                      # a row of each of two sequences is not one sequence of two rows
        block.forward(x[:2], positions[:2], cache=(held, table, ints(1, 1)))
    assert block.forward(x[:0], positions[:0], ints(0), cache=(held, table[:0], table[:0, 0])).shape == (0, 64)


@pytest.mark.gpu
def test_the_shortest_run_of_the_command():
    assert len(at.main(["--steps", "1", "--rows", "3", "--width", "64", "--heads", "2", "--kv-heads", "1"])) == 1


@pytest.mark.gpu
@pytest.mark.parametrize("packed", [False, True])
def test_prompts_in_a_graph(server, packed):
    block, cache, table = server
    x, positions = torch.randn(20, 64, device="cuda"), torch.arange(20, device="cuda")
    s, table, lens = (ints(0, 9, 20), table, ints(9, 11)) if packed else (None, table[:1], ints(20))
    held, eager = cache(), cache()
    block.forward(x, positions, s, cache=(eager, table, lens))   # (what a first call sets up is not captured)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        y = block.forward(x, positions, s, cache=(held, table, lens))
    for a, b in zip(held, eager):
        a.copy_(b)
    for more in (0, 0, 1, 0):                            # in the third replay a sequence holds an older token
        x.copy_(torch.randn_like(x))
        lens[0] += more
        g.replay()
        torch.cuda.synchronize()
        want = block.forward(x, positions, s, cache=(eager, table, lens))
        assert torch.equal(y.isnan(), want.isnan()) and bool(y.isnan().any()) == (more == 1) and torch.equal(y.nan_to_num(), want.nan_to_num())
        assert all(torch.equal(a, b) for a, b in zip(held, eager))
        lens[0] -= more

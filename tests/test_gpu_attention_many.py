"""Attention over lists of many sequences: where each has its tiles, whatever their lengths, and that the longest list takes no longer than its rows do."""
import numpy as np
import pytest
import torch

import layer_oracle as lo
from paper_2401_14110_amd import binding as lb
from test_gpu_attention import check
from test_gpu_layernorm import near


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("count,longest,extra", [(63, 200, 0), (64, 150, 3), (65, 150, 0), (65, 3, 130), (129, 140, 5), (300, 130, 1), (700, 4, 0), (4097, 2, 9)])
def test_lengths_of_all_kinds(count, longest, extra, dtype):
    rng = np.random.default_rng(count + longest)
    lens, lens_k = (rng.integers(0, longest + 1, count) for _ in range(2))
    lens[rng.random(count) < 0.2], lens_k[rng.random(count) < 0.2] = 0, 0            # and runs of empty ones
    lens[count // 3:count // 2] = 0
    lens[-1], lens_k[0] = 129, 257
    check([int(n) for n in lens], [int(n) for n in lens_k], 2, 1, 16, True, dtype, extra=extra)


@pytest.mark.gpu
def test_more_sequences_than_rows():
    g = torch.Generator(device="cuda").manual_seed(0)
    q, G = (torch.randn(5, 2, 32, device="cuda", generator=g).bfloat16() for _ in range(2))
    s = torch.zeros(100001, dtype=torch.int32, device="cuda")
    s[777:], s[50000:] = 2, 5                            # sequences 776 of two rows and 49999 of three
    o, lse = lb.attention(q, q, q, starts=s, want_stats=True)
    few = torch.tensor([0, 2, 5], dtype=torch.int32, device="cuda")
    wo, wl = lb.attention(q, q, q, starts=few, want_stats=True)
    assert torch.equal(o, wo) and torch.equal(lse, wl)
    for a, b in zip(lb.attention_bwd(G, q, q, q, o, lse, starts=s), lb.attention_bwd(G, q, q, q, wo, wl, starts=few)):
        assert torch.equal(a, b)


@pytest.mark.gpu
def test_the_longest_list():
    """2^20 sequences of one token each: the value itself, but for w v and 1 / w, whose weight w is near 1: 8 roundings."""
    count, H = 1 << 20, 7
    v = torch.randn(count, H, 8, device="cuda", generator=torch.Generator(device="cuda").manual_seed(1))
    s = torch.arange(count + 1, dtype=torch.int32, device="cuda")
    o, lse = lb.attention(v, v, v, starts=s, want_stats=True)
    want = v.double()
    assert ((o.double() - want).abs() <= 8 * lo.U * want.abs() + 2.0 ** -126).all()
    near(lse[::997], 8 ** -0.5 * (want * want).sum(-1)[::997].cpu().numpy(), 20 * lo.U * (1 + (want * want).sum(-1)[::997].cpu().numpy()), "f32")
    G = torch.randn(v.shape, device="cuda", generator=torch.Generator(device="cuda").manual_seed(2))
    dq, dk, dv = lb.attention_bwd(G, v, v, v, o, lse, starts=s)
    assert not dq.any() and not dk.any()
    # a weight of e^(score - lse): both off by a few units of their size
    near(dv[::997], G.double()[::997].cpu().numpy(), 60 * lo.U * ((1 + (want * want).sum(-1)[::997, :, None]) * G.double()[::997].abs()).cpu().numpy() + 2.0 ** -126, "f32")
    with pytest.raises(lb.LbaError):                     # (2^20 + 2^13) * 8 tiles
        lb.attention(v[:, :1].expand(-1, 8, -1), v[:, :1], v[:, :1], starts=s)

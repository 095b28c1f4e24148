"""Rotary positions and their gradient against the formula in 64 bits: layouts, part of the head, odd widths, views, far positions, types;
in place, on streams and in replayed graphs; refusals."""
import ctypes

import numpy as np
import pytest
import torch

import attention_oracle as ao
from paper_2401_14110_amd import binding as lb
from test_gpu_layernorm import DEV, DT, dev, host, near, values


def frequencies(pairs, base=10000.0):
    return base ** (-np.arange(pairs) / max(pairs, 1))


def check(x, positions, freq, interleaved, gain, dtype, tx=None, pos_type=torch.int64):
    tp, tf = torch.from_numpy(positions).to(DEV, pos_type), torch.from_numpy(freq).to(DEV)
    tx = dev(x, dtype) if tx is None else tx
    for call, sign in ((lb.rope, 1.0), (lb.rope_bwd, -1.0)):
        want, tol = ao.rope(x, positions, freq, interleaved, gain, sign)
        got = call(tx, tp, tf, interleaved=interleaved, gain=gain)
        assert got.dtype == DT[dtype] and got.shape == tx.shape
        near(got, want, tol, dtype)
        R = 2 * len(freq)
        assert torch.equal(got[..., R:], tx[..., R:])                                # copied as it is


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("T,H,D,R", [(1, 1, 2, 2), (1, 12, 64, 64), (3, 5, 7, 6), (9, 40, 128, 128), (33, 3, 80, 32), (5, 2, 83, 82), (17, 4, 128, 0), (4, 7, 96, 2),
                                     (70, 1, 256, 256), (5, 3, 1024, 1024), (6, 2, 1023, 514), (11, 9, 65, 30), (2, 64, 40, 38)])
def test_against_the_formula(T, H, D, R, interleaved, dtype):
    rng = np.random.default_rng(T * 1000 + D)
    x = values(rng, (T, H, D), dtype)
    check(x, rng.integers(0, 5000, T), frequencies(R // 2), interleaved, 1.0, dtype)
    check(x, rng.integers(-500, 131072, T), frequencies(R // 2, 5e5) / 4.0, interleaved, 1.1386, dtype, pos_type=torch.int32)


@pytest.mark.gpu
def test_far_positions():
    x = values(np.random.default_rng(1), (6, 3, 64), "f32")
    check(x, np.array([0, 1, 2 ** 20 + 1, 2 ** 31 - 1, 2 ** 40 + 7, -2 ** 33]), frequencies(32), False, 1.0, "f32")


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_views_and_in_place(dtype):
    rng = np.random.default_rng(2)
    T, H, KV, D = 21, 6, 2, 48
    qkv = dev(values(rng, (T, H + 2 * KV, D), dtype), dtype)
    p, f = torch.arange(T, device=DEV), torch.from_numpy(frequencies(20)).to(DEV)
    part = qkv[:, :H + KV]
    want = lb.rope(part.clone(), p, f)
    before = qkv.clone()
    assert torch.equal(lb.rope(part, p, f), want) and torch.equal(qkv, before)
    assert lb.rope(part, p, f, out=part) is part
    assert torch.equal(part, want) and torch.equal(qkv[:, H + KV:], before[:, H + KV:])
    batch = before.view(3, 7, H + 2 * KV, D)[:, :, :H]                               # leading axes that are one in memory
    assert torch.equal(lb.rope(batch, p.view(3, 7), f), want[:, :H].reshape(3, 7, H, D))
    turned = before[:, :H].transpose(0, 1).contiguous().transpose(0, 1)              # heads outermost
    assert torch.equal(lb.rope(turned, p, f), want[:, :H])
    odd = before[:, :H].permute(2, 0, 1).contiguous().permute(1, 2, 0)               # D not along memory: copied
    assert torch.equal(lb.rope(odd, p, f), want[:, :H])
    one = before[:, :1].expand(T, 5, D)                                              # a broadcast input
    assert torch.equal(lb.rope(one, p, f), want[:, :1].expand(T, 5, D))
    e = torch.empty(0, 4, 8, device=DEV)
    assert lb.rope(e, p[:0], f[:4]).shape == (0, 4, 8)


@pytest.mark.gpu
def test_what_is_copied_keeps_its_bits():
    bits = torch.tensor([1, 0x7FC1, 0x7F80, -0x7FFF, 0x0080, 3, 5, 7, 9, 11, 13], dtype=torch.int16, device=DEV)
    x = bits.view(torch.bfloat16).repeat(3, 2, 1)
    y = lb.rope(x, torch.arange(3, device=DEV), torch.ones(0, dtype=torch.float64, device=DEV))
    assert torch.equal(y.view(torch.int16), x.view(torch.int16))


@pytest.mark.gpu
def test_streams_and_replays():
    x = torch.randn(40, 4, 64, device=DEV)
    p, f = torch.arange(40, device=DEV, dtype=torch.int32), torch.from_numpy(frequencies(32)).to(DEV)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    y = lb.rope(x, p, f, stream=s)
    s.synchronize()
    assert torch.equal(y, lb.rope(x, p, f))
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out = lb.rope(x, p, f)
        back = lb.rope_bwd(out, p, f)
    for k in range(3):
        x.copy_(torch.randn_like(x))
        p.add_(1000 * k)
        g.replay()
        torch.cuda.synchronize()
        want = lb.rope(x, p, f)
        assert torch.equal(out, want) and torch.equal(back, lb.rope_bwd(want, p, f))


@pytest.mark.gpu
def test_offsets_beyond_32_bits():
    T, row = 70001, 65536
    x = torch.zeros((T, row), dtype=torch.bfloat16, device=DEV)[:, :64].view(T, 2, 32)
    x[-1] = 1.0
    p, f = torch.full((T,), 3, device=DEV), torch.from_numpy(frequencies(16)).to(DEV)
    y = lb.rope(x, p, f)
    want, tol = ao.rope(np.ones((1, 2, 32)), np.array([3]), frequencies(16), False, 1.0)
    near(y[-1:], want, tol, "bf16")
    assert not y[:-1].any()


def test_refusals():
    P, s = ctypes.c_void_p(0x1000), lb.lba_strides(64, 32)
    call = lambda **k: lb.lba_rope(*{**dict(X=P, xa=s, t=0, pos=P, bits=64, f=P, pairs=16, i=0, gain=1.0, Y=P, ya=s, T=4, H=2, D=32), **k}.values())  # noqa: E731
    assert call(X=None) == lb.ERR_NULL and call(Y=None) == lb.ERR_NULL and call(pos=None) == lb.ERR_NULL and call(f=None) == lb.ERR_NULL
    assert call(pairs=17) == lb.ERR_SHAPE and call(pairs=-1) == lb.ERR_SHAPE and call(T=-1) == lb.ERR_SHAPE and call(T=1 << 31) == lb.ERR_SHAPE
    assert call(H=65536) == lb.ERR_SHAPE and call(D=1025) == lb.ERR_SHAPE and call(xa=lb.lba_strides(-1, 1)) == lb.ERR_SHAPE
    assert call(t=2) == lb.ERR_UNSUPPORTED and call(bits=16) == lb.ERR_UNSUPPORTED
    assert call(T=0, X=None) == lb.OK and call(H=0, X=None) == lb.OK and call(D=0, pairs=0, X=None) == lb.OK
    assert lb.lba_rope_bwd(None, s, 0, P, 64, P, 16, 0, 1.0, P, s, 4, 2, 32) == lb.ERR_NULL


@pytest.mark.gpu
def test_refusals_of_tensors():
    x, p, f = torch.randn(4, 2, 8, device=DEV), torch.arange(4, device=DEV), torch.ones(4, dtype=torch.float64, device=DEV)
    for bad in (lambda: lb.rope(x, p.float(), f), lambda: lb.rope(x, p[:3], f), lambda: lb.rope(x, p, f.float()), lambda: lb.rope(x, p, torch.cat([f, f])),
                lambda: lb.rope(x[0], p, f), lambda: lb.rope(x, p, f, out=x[:, :1].expand(4, 2, 8)), lambda: lb.rope(x, p, f, out=x.bfloat16()),
                lambda: lb.rope(x, p, f, out=x.transpose(1, 2).contiguous().transpose(1, 2))):
        with pytest.raises(ValueError):
            bad()
    for bad in (lambda: lb.rope(x.half(), p, f), lambda: lb.rope(x.cpu(), p, f)):
        with pytest.raises(TypeError):
            bad()

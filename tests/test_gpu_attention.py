"""Attention over packed sequences and its gradients against the formulas in 64 bits: lengths around the tiles' edges, empty sequences, queries that
see nothing, grouped heads, widths of every kind, both types; views, streams and replays; what is hidden; refusals."""
import ctypes

import numpy as np
import pytest
import torch

import attention_oracle as ao
import layer_oracle as lo
from paper_2401_14110_amd import binding as lb
from test_gpu_layernorm import DEV, DT, dev, host, near, values


def ints(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def starts(lens, first=0):
    return ints(list(np.cumsum([first] + list(lens))))


def check(lens, lens_k, H, KV, D, causal, dtype, train=True, extra=0, scale=None, spread=1.0, out_type=None):
    """One call each way; `extra` rows of no sequence before and behind."""
    rng = np.random.default_rng(sum(lens) * 131 + D * 7 + H)
    T, Tk = sum(lens) + 2 * extra, sum(lens_k) + 2 * extra
    q, k, v, G = (values(rng, s, dtype, c) for s, c in (((T, H, D), spread), ((Tk, KV, D), spread), ((Tk, KV, D), 1.0), ((T, H, D), 1.0)))
    sc = D ** -0.5 if scale is None else scale
    want = ao.packed(q, k, v, lens, lens_k, causal, float(np.float32(sc)), dtype, G if train else None, extra, extra)
    tq, tk, tv, tG = (dev(x, dtype) for x in (q, k, v, G))
    kw = dict(starts=starts(lens, extra), starts_k=starts(lens_k, extra), causal=causal, scale=scale)
    o, lse = lb.attention(tq, tk, tv, want_stats=True, **kw)
    near(o, *want["o"], dtype)
    none = np.isinf(want["lse"][0])
    assert np.array_equal(host(lse)[none], want["lse"][0][none])
    near(torch.where(torch.from_numpy(none).to(DEV), 0.0, lse), np.where(none, 0.0, want["lse"][0]), want["lse"][1], "f32")
    if train:
        for got, w in zip(lb.attention_bwd(tG, tq, tk, tv, o, lse, **kw), ("dq", "dk", "dv")):
            assert got.dtype == DT[dtype]
            near(got, *want[w], dtype)
    return want, (tq, tk, tv, tG, o, lse, kw)


SHAPES = [([1], [1], 1, 1, 1), ([24], [24], 12, 12, 64), ([1, 2, 3], [1, 2, 3], 2, 1, 7), ([31, 0, 33], [31, 0, 33], 2, 2, 16), ([32, 65], [32, 65], 3, 1, 33),
          ([127, 1, 130], [127, 1, 130], 4, 2, 80), ([200], [200], 2, 1, 83), ([129, 64], [129, 64], 2, 2, 96), ([300, 5], [300, 5], 4, 1, 128),
          ([257], [257], 1, 1, 127), ([63, 128, 64], [63, 128, 64], 2, 1, 64),
          # keys behind the queries' past, fewer keys than queries (the first queries see nothing), keys or queries of none
          ([5, 17], [70, 17], 2, 1, 64), ([70], [33], 2, 2, 40), ([140, 9], [1, 200], 2, 1, 128), ([6, 0, 8], [0, 9, 8], 2, 2, 24), ([1], [513], 8, 1, 128), ([513], [1], 2, 2, 32)]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "-".join(str(x) for x in s).replace(" ", ""))
def test_against_the_formulas(shape, causal, dtype):
    check(*shape, causal, dtype)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_longer_sequences(dtype):
    check([700, 1100], [700, 1100], 2, 1, 64, True, dtype)
    check([1025], [1500], 2, 1, 128, False, dtype)
    check([90, 333, 1, 258], [90, 333, 1, 258], 6, 2, 72, True, dtype, extra=37)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_large_scores(dtype):
    # scores of hundreds: weights of 0 and 1, a maximum that moves; and equal scores
    check([150], [150], 2, 1, 64, True, dtype, spread=6.0)
    check([150], [150], 2, 1, 64, False, dtype, scale=0.0)
    check([150], [150], 2, 1, 64, True, dtype, scale=-0.25)


@pytest.mark.gpu
def test_rising_scores():
    """Keys that grow along the sequence: the running maximum moves at every tile; and fall: it never does."""
    rng = np.random.default_rng(5)
    for grow in (np.linspace(0, 30, 400), np.linspace(30, 0, 400)):
        q = np.abs(values(rng, (400, 1, 32), "f32"))
        k = (values(rng, (400, 1, 32), "f32") * 0.1 + grow[:, None, None]).astype(np.float32)
        v = values(rng, (400, 1, 32), "f32")
        for dtype in ("f32", "bf16"):
            a, b, c = (lo.bf16(t) if dtype == "bf16" else t for t in (q, k, v))
            want = ao.packed(a, b, c, [400], [400], False, float(np.float32(32 ** -0.5)), dtype)
            near(lb.attention(dev(a, dtype), dev(b, dtype), dev(c, dtype), causal=False), *want["o"], dtype)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_output_types(dtype):
    want, (q, k, v, _, o, _, kw) = check([65, 130, 3], [65, 130, 3], 4, 2, 64, True, dtype, train=False)
    for out in ("f32", "bf16"):
        near(lb.attention(q, k, v, out_dtype=DT[out], **kw), *want["o"], out)
    for fmt in ((4, 3, 7 + 6), (3, 4, 3 + 2), (5, 2, 15)):
        codes = lb.attention(q, k, v, out_dtype=torch.uint8, out_fmt=fmt, **kw)
        lo.check_codes(codes.cpu().numpy(), want["o"][0], want["o"][1] + 2 * lo.U * np.abs(want["o"][0]), fmt)


@pytest.mark.gpu
@pytest.mark.parametrize("lens,H,KV,D,causal", [([1], 1, 1, 1, True), ([33, 0, 130], 4, 2, 64, True), ([200, 65], 6, 2, 83, False), ([300], 2, 1, 128, True), ([2, 129], 3, 3, 96, True),
                                               ([70], 2, 2, 116, True)])
def test_float32_outputs_of_bfloat16_inputs(lens, H, KV, D, causal):
    """Weights are not rounded then: the bounds are those of float32."""
    g = torch.Generator(device="cuda").manual_seed(sum(lens))
    q, k, v = (torch.randn(sum(lens), h, D, device="cuda", generator=g).bfloat16() for h in (H, KV, KV))
    s = torch.tensor(np.cumsum([0] + lens), dtype=torch.int32).cuda()
    want = ao.packed(*(t.double().cpu().numpy() for t in (q, k, v)), lens, lens, causal, float(np.float32(D ** -0.5)), "f32")
    got = lb.attention(q, k, v, starts=s, causal=causal, out_dtype=torch.float32)
    near(got, *want["o"], "o")


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("lens,lens_k,causal", [([1, 5, 1, 200], [1, 5, 1, 200], True), ([3, 140], [1, 1], False), ([4, 70], [1, 1], True), ([9, 130], [4, 129], True)])
def test_a_query_that_sees_one_key_has_no_gradient_of_its_score(lens, lens_k, causal, dtype):
    g = torch.Generator(device="cuda").manual_seed(1)
    q = torch.randn(sum(lens), 4, 64, device="cuda", generator=g).to(DT[dtype])
    k, v = (torch.randn(sum(lens_k), 2, 64, device="cuda", generator=g).to(DT[dtype]) for _ in range(2))
    s, sk = (torch.tensor(np.cumsum([0] + n), dtype=torch.int32).cuda() for n in (lens, lens_k))
    o, lse = lb.attention(q, k, v, starts=s, starts_k=sk, causal=causal, want_stats=True)
    G = torch.randn(q.shape, device="cuda", generator=g).to(DT[dtype])
    dq, dk, dv = lb.attention_bwd(G, q, k, v, o, lse, starts=s, starts_k=sk, causal=causal)
    a = b = 0
    for n, m in zip(lens, lens_k):
        seen = [min(m, max(0, i + m - n + 1)) if causal else m for i in range(n)]
        rows = torch.tensor([a + i for i in range(n) if seen[i] == 1], dtype=torch.long, device="cuda")
        assert len(rows) and not dq[rows].any()
        assert m > 1 or (not dk[b:b + 1].any() and bool(dv[b:b + 1].any()))
        a, b = a + n, b + m
    # what the lone query leaves to its key's gradient: nothing, of whatever size its own gradient is
    lone = torch.tensor(np.cumsum([0] + lens[:-1]) + np.maximum(0, np.array(lens) - np.array(lens_k)), device="cuda")
    if causal:
        G[lone] *= 1024.0
        assert torch.equal(lb.attention_bwd(G, q, k, v, o, lse, starts=s, starts_k=sk)[1], dk)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_views_batches_and_given_outputs(dtype):
    rng = np.random.default_rng(3)
    B, L, H, KV, D = 3, 70, 4, 2, 48
    qkv = dev(values(rng, (B * L, H + 2 * KV, D), dtype), dtype)
    G = dev(values(rng, (B * L, H, D), dtype), dtype)
    q, k, v = qkv[:, :H], qkv[:, H:H + KV], qkv[:, H + KV:]
    s = starts([L] * B)
    o, lse = lb.attention(q.contiguous(), k.contiguous(), v.contiguous(), starts=s, want_stats=True)
    grads = lb.attention_bwd(G, q.contiguous(), k.contiguous(), v.contiguous(), o, lse, starts=s)
    got, st = lb.attention(q, k, v, starts=s, want_stats=True)
    assert torch.equal(got, o) and torch.equal(st, lse)
    # gradients straight into one tensor
    d = torch.full_like(qkv, float("nan"))
    back = lb.attention_bwd(G, q, k, v, o, lse, starts=s, out=(d[:, :H], d[:, H:H + KV], d[:, H + KV:]))
    assert back[0].data_ptr() == d.data_ptr() and torch.equal(d, torch.cat(grads, 1))
    # equal lengths as a batch
    four = lambda t: t.view((B, L) + t.shape[1:])  # noqa: E731
    q4, k4, v4 = (t.unflatten(0, (B, L)) for t in (q, k, v))
    o4, l4 = lb.attention(q4, k4, v4, want_stats=True)
    assert torch.equal(o4, four(o)) and torch.equal(l4, four(lse))
    for a, b in zip(lb.attention_bwd(four(G), q4, k4, v4, o4, l4), grads):
        assert torch.equal(a, four(b))
    # heads outermost, D not along memory, broadcast keys
    turned = [t.transpose(0, 1).contiguous().transpose(0, 1) for t in (q, k, v)]
    assert torch.equal(lb.attention(*turned, starts=s), o)
    odd = [t.permute(2, 0, 1).contiguous().permute(1, 2, 0) for t in (q, k, v)]
    assert torch.equal(lb.attention(*odd, starts=s), o)
    one = k[:, :1].expand(-1, 2, -1)
    assert torch.equal(lb.attention(q, one, v, starts=s), lb.attention(q, one.contiguous(), v, starts=s))
    # one sequence
    assert torch.equal(lb.attention(q[:L], k[:L], v[:L]), o[:L])


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_rows_of_no_sequence(dtype):
    rng = np.random.default_rng(4)
    T, H, D, lens = 300, 2, 64, [70, 0, 65]
    q, k, v, G = (dev(values(rng, (T, H, D), dtype), dtype) for _ in range(4))
    for t in (q, k, v, G):
        t[:11] = float("nan")
        t[11 + sum(lens):] = float("inf")
    s = starts(lens, 11)
    i = slice(11, 11 + sum(lens))
    o, lse = lb.attention(q, k, v, starts=s, want_stats=True)
    inner = [t[i].contiguous() for t in (q, k, v, G)]
    wo, wl = lb.attention(*inner[:3], starts=starts(lens), want_stats=True)
    assert torch.equal(o[i], wo) and not o[:11].any() and not o[i.stop:].any()
    assert torch.equal(lse[i], wl) and (lse[:11] == -float("inf")).all() and (lse[i.stop:] == -float("inf")).all()
    want = lb.attention_bwd(inner[3], *inner[:3], wo, wl, starts=starts(lens))
    for a, b in zip(lb.attention_bwd(G, q, k, v, o, lse, starts=s), want):
        assert torch.equal(a[i], b) and not a[:11].any() and not a[i.stop:].any()
    given = torch.full_like(o, 7.0)
    assert lb.attention(q, k, v, starts=s, out=given) is given
    assert torch.equal(given[i], wo) and (given[:11] == 7).all() and (given[i.stop:] == 7).all()
    held = [torch.full_like(t, 7.0) for t in (q, k, v)]
    for a, b in zip(lb.attention_bwd(G, q, k, v, o, lse, starts=s, out=held), want):
        assert torch.equal(a[i], b) and (a[:11] == 7).all() and (a[i.stop:] == 7).all()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("where", [0, 5, 40, 63, 64, 100, 149])
def test_what_later_tokens_hold_does_not_matter(where, dtype):
    """Infinities and NaN in a token's key and value: the queries before it, and their gradients, are as if it were not there."""
    rng = np.random.default_rng(6)
    n, H, KV, D = 150, 2, 1, 64
    q, k, v, G = (dev(values(rng, (n, h, D), dtype), dtype) for h in (H, KV, KV, H))
    G[where:] = 0.0
    clean = lb.attention(q[:where], k[:where], v[:where], want_stats=True)
    clean_d = lb.attention_bwd(G[:where], q[:where], k[:where], v[:where], *clean)
    k[where, 0, ::3], k[where, 0, 1::3] = float("nan"), float("inf")
    v[where, 0, ::2], v[where, 0, 1::2] = float("-inf"), float("nan")
    o, lse = lb.attention(q, k, v, want_stats=True)
    near(o[:where], host(clean[0]), 8 * lo.U * (1 + np.abs(host(clean[0]))) + (2.0 ** -8 if dtype == "bf16" else 0) * 4, dtype)
    assert o[:where].isfinite().all() and lse[:where].isfinite().all() and not o[where:].isfinite().any()
    dq, dk, dv = lb.attention_bwd(G, q, k, v, o, lse)
    assert dq[:where].isfinite().all()
    if where:
        assert (dq[:where].float() - clean_d[0].float()).abs().max() <= (2.0 ** -5 if dtype == "bf16" else 2.0 ** -18)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("where", [0, 31, 32, 64, 149])
def test_what_earlier_queries_hold_does_not_matter_to_later_keys(where, dtype):
    """Infinities in a query and its gradient reach only the keys that it sees."""
    rng = np.random.default_rng(7)
    n, D = 150, 64
    q, k, v, G = (dev(values(rng, (n, 1, D), dtype), dtype) for _ in range(4))
    o, lse = lb.attention(q, k, v, want_stats=True)
    clean = lb.attention_bwd(G, q, k, v, o, lse)
    q[where, 0, ::3], G[where, 0, ::2] = float("inf"), float("nan")
    _, dk, dv = lb.attention_bwd(G, q, k, v, o, lse)
    tol = 2.0 ** -5 if dtype == "bf16" else 2.0 ** -18
    for a, b in ((dk, clean[1]), (dv, clean[2])):
        assert a[where + 1:].isfinite().all()
        if where + 1 < n:
            assert (a[where + 1:].float() - b[where + 1:].float()).abs().max() <= tol


@pytest.mark.gpu
def test_a_seen_infinity():
    v = torch.zeros(70, 1, 32, device=DEV)
    v[3, 0, 1], v[3, 0, 2], v[66, 0, 2] = float("inf"), float("-inf"), float("inf")
    q = torch.zeros(70, 1, 32, device=DEV)
    for dtype in ("f32", "bf16"):
        o = lb.attention(q.to(DT[dtype]), q.to(DT[dtype]), v.to(DT[dtype])).float()
        assert (o[:3] == 0).all() and (o[3:, 0, 1] == float("inf")).all() and (o[3:66, 0, 2] == float("-inf")).all() and o[66:, 0, 2].isnan().all()
        assert (o[:, 0, 3:] == 0).all() and (o[:, 0, 0] == 0).all()


@pytest.mark.gpu
def test_differences():
    rng = np.random.default_rng(8)
    lens, H, KV, D, eps = [37, 5], 4, 2, 16, 2.0 ** -6
    T = sum(lens)
    q, k, v, G = (values(rng, (T, h, D), "f32") for h in (H, KV, KV, H))
    s = starts(lens)
    loss = lambda *a: float((G * host(lb.attention(*map(dev, a), starts=s))).sum())  # noqa: E731
    o, lse = lb.attention(dev(q), dev(k), dev(v), starts=s, want_stats=True)
    grads = lb.attention_bwd(dev(G), dev(q), dev(k), dev(v), o, lse, starts=s)
    for i, g in enumerate(grads):
        args = [q, k, v]
        step = np.float32(eps) * np.sign(rng.standard_normal(args[i].shape)).astype(np.float32)
        up, down = ([a + c * step if j == i else a for j, a in enumerate(args)] for c in (np.float32(1), np.float32(-1)))
        slope = (loss(*up) - loss(*down)) / (2 * eps)
        # third-order error eps^2 of T H D terms of size |G|, added at random: below 1e-2 of the scale sqrt(T H D)
        assert abs(slope - float((host(g) * step / eps).sum())) <= 1e-2 * np.sqrt(T * H * D), i


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_streams_replays_and_equal_bits(dtype):
    lens = [100, 33, 260]
    _, (q, k, v, G, o, lse, kw) = check(lens, lens, 4, 2, 64, True, dtype)
    want = lb.attention_bwd(G, q, k, v, o, lse, **kw)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    o2, l2 = lb.attention(q, k, v, want_stats=True, stream=s, **kw)
    d2 = lb.attention_bwd(G, q, k, v, o2, l2, stream=s, **kw)
    s.synchronize()
    assert torch.equal(o2, o) and torch.equal(l2, lse) and all(torch.equal(a, b) for a, b in zip(d2, want))
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        go, gl = lb.attention(q, k, v, want_stats=True, **kw)
        gd = lb.attention_bwd(G, q, k, v, go, gl, **kw)
    # other lengths in the same list, and other values, at each replay
    for lens in ([100, 33, 260], [1, 390, 0], [393, 0, 0], [50, 60, 70]):
        kw["starts"].copy_(starts(lens))
        kw["starts_k"].copy_(starts(lens))
        q.copy_(torch.randn_like(q))
        g.replay()
        torch.cuda.synchronize()
        eo, el = lb.attention(q, k, v, want_stats=True, **kw)
        assert torch.equal(go, eo) and torch.equal(gl, el)
        for a, b in zip(gd, lb.attention_bwd(G, q, k, v, eo, el, **kw)):
            assert torch.equal(a, b)


@pytest.mark.gpu
def test_lists_that_break_the_contract_stay_inside():
    """Starts that fall, are negative or point behind the tensors: whatever comes out, nothing outside the tensors is touched."""
    T, H, D = 90, 2, 32
    q, k, v, G = (torch.randn(T, H, D, device=DEV) for _ in range(4))
    for bad in ([0, 60, 30, 90], [-50, 20, 1000], [2 ** 31 - 1, -2 ** 31, 5], [90, 0], [0, 2 ** 31 - 1]):
        s = ints(bad)
        held = [torch.full((T + 64, H, D), 7.0, device=DEV) for _ in range(4)]
        out = [t[32:32 + T] for t in held]
        lb.attention(q, k, v, starts=s, out=out[0])
        o, lse = lb.attention(q, k, v, starts=s, want_stats=True)
        lb.attention_bwd(G, q, k, v, o, lse, starts=s, out=out[1:])
        torch.cuda.synchronize()
        assert all((t[:32] == 7).all() and (t[32 + T:] == 7).all() for t in held), bad


@pytest.mark.gpu
def test_many_sequences():
    rng = np.random.default_rng(9)
    lens = [int(n) for n in rng.integers(0, 6, 700)]
    check(lens, lens, 2, 1, 16, True, "bf16")
    count = 5000                                         # one token each: the value itself, but for w v and 1 / w, whose weight w is near 1: 8 roundings
    v = torch.randn(count, 2, 8, device=DEV)
    near(lb.attention(v, v, v, starts=torch.arange(count + 1, dtype=torch.int32, device=DEV)), host(v), 8 * lo.U * np.abs(host(v)), "f32")


@pytest.mark.gpu
def test_offsets_beyond_32_bits():
    T, row = 70001, 65536
    big = torch.zeros((T, row), dtype=torch.bfloat16, device=DEV)
    x = big[:, :64].view(T, 1, 64)
    n = 200
    x[-n:] = torch.randn(n, 1, 64, device=DEV).bfloat16()
    s = ints([T - n, T])
    c = x[-n:].contiguous()
    o, lse = lb.attention(x, x, x, starts=s, want_stats=True)
    wo, wl = lb.attention(c, c, c, want_stats=True)
    assert torch.equal(o[-n:], wo)
    G = torch.randn(T, 1, 64, device=DEV).bfloat16()
    d = [big[:, i:i + 64].view(T, 1, 64) for i in (128, 256, 384)]
    lb.attention_bwd(G, x, x, x, o, lse, starts=s, out=d)
    for a, b in zip(d, lb.attention_bwd(G[-n:].contiguous(), c, c, c, wo, wl)):
        assert torch.equal(a[-n:], b) and not a[:-n].any()


@pytest.mark.gpu
def test_nothing_to_do():
    e, k = torch.empty(0, 4, 16, device=DEV), torch.randn(6, 2, 16, device=DEV)
    o, lse = lb.attention(e, e[:, :2], e[:, :2], want_stats=True)
    assert o.shape == (0, 4, 16) and lse.shape == (0, 4)
    assert all(t.shape[0] == 0 for t in lb.attention_bwd(e, e, e[:, :2], e[:, :2], o, lse))
    # queries without keys, keys without queries
    q = torch.randn(6, 4, 16, device=DEV)
    none = torch.empty(0, 2, 16, device=DEV)
    o, lse = lb.attention(q, none, none, starts=ints([0, 6]), starts_k=ints([0, 0]), want_stats=True)
    assert not o.any() and (lse == -float("inf")).all()
    dq, dk, dv = lb.attention_bwd(q, q, none, none, o, lse, starts=ints([0, 6]), starts_k=ints([0, 0]))
    assert not dq.any() and dk.shape == (0, 2, 16)
    dq, dk, dv = lb.attention_bwd(e, e, k, k, e, torch.empty(0, 4, device=DEV), starts=ints([0, 0]), starts_k=ints([0, 6]))
    assert not dk.any() and not dv.any()
    assert not lb.attention(q, k, k, starts=ints([0])).any()                         # no sequences


def desc(**k):
    s = lb.lba_strides(64, 16)
    d = dict(T=8, Tk=8, count=1, starts=None, starts_k=None, H=4, KV=2, D=16, type=0, causal=1, clear=0, scale=0.25, q=s, k=s, v=s)
    return lb.lba_attn(*{**d, **k}.values())


def test_refusals():
    P, W, f, s = ctypes.c_void_p(0x1000), ctypes.c_void_p(0x2000), (4, 3, 7), lb.lba_strides(64, 16)
    call = lambda a=None, **k: lb.lba_attention(*{**dict(a=a or desc(), Q=P, K=P, V=P, O=P, t=0, f=f, lse=None, ws=None, n=0), **k}.values())  # noqa: E731
    need = lb.lba_attention_bwd_workspace_bytes(desc())
    assert need >= 8 * 4 * 4
    back = lambda a=None, **k: lb.lba_attention_bwd(*{**dict(a=a or desc(), G=P, Q=P, K=P, V=P, O=P, lse=P, dQ=P, qa=s, dK=P, ka=s, dV=P, va=s, ws=W, n=need), **k}.values())  # noqa: E731
    for fn in (call, back):
        for bad in (dict(T=-1), dict(T=1 << 31), dict(Tk=1 << 31), dict(D=0), dict(D=129), dict(H=5), dict(KV=0), dict(KV=3), dict(count=-1), dict(count=3), dict(H=65536, KV=1),
                    dict(count=(1 << 20) + 1, starts=P), dict(q=lb.lba_strides(-1, 0)), dict(k=lb.lba_strides(0, -1)), dict(v=lb.lba_strides(-1, 0)), dict(count=0)):
            assert fn(desc(**bad)) == lb.ERR_SHAPE, bad
        assert fn(desc(type=2)) == lb.ERR_UNSUPPORTED and fn(desc(starts_k=P)) == lb.ERR_NULL
        assert fn(Q=None) == lb.ERR_NULL and fn(K=None) == lb.ERR_NULL and fn(V=None) == lb.ERR_NULL and fn(O=None) == lb.ERR_NULL
        assert fn(desc(T=0, Tk=0), Q=None, K=None, V=None, O=None) == lb.OK
    assert call(t=3) == lb.ERR_UNSUPPORTED and call(t=2, f=(1, 6, 0)) == lb.ERR_FORMAT
    for w in ("G", "lse", "dQ", "dK", "dV", "ws"):
        assert back(**{w: None}) == lb.ERR_NULL, w
    assert back(ws=ctypes.c_void_p(0x2010)) == lb.ERR_ALIGN and back(n=need - 1) == lb.ERR_SHAPE and back(ka=lb.lba_strides(-1, 1)) == lb.ERR_SHAPE


@pytest.mark.gpu
def test_refusals_of_tensors():
    q, k = torch.randn(8, 4, 16, device=DEV), torch.randn(8, 2, 16, device=DEV)
    s = ints([0, 8])
    for bad in (lambda: lb.attention(q, k, k[:7]), lambda: lb.attention(q, k[..., :8], k[..., :8]), lambda: lb.attention(q[:, :3], k, k), lambda: lb.attention(q, k, k, starts=s.long()),
                lambda: lb.attention(q, k, k, starts_k=s), lambda: lb.attention(q, k[:4], k[:4], starts=s), lambda: lb.attention(q, k, k, starts=s, starts_k=ints([0, 4, 8])),
                lambda: lb.attention(q.view(2, 4, 4, 16), k, k), lambda: lb.attention(q, k, k, out_dtype=torch.uint8), lambda: lb.attention(q, k, k, out=q[:4]),
                lambda: lb.attention(torch.randn(4, 2, 130, device=DEV), torch.randn(4, 2, 130, device=DEV), torch.randn(4, 2, 130, device=DEV)),
                lambda: lb.attention(q.view(2, 4, 4, 16), k.view(2, 4, 2, 16), k.view(2, 4, 2, 16), starts=s), lambda: lb.attention(q[0], k[0], k[0])):
        with pytest.raises(ValueError):
            bad()
    o, lse = lb.attention(q, k, k, want_stats=True)
    one = torch.zeros(8, 1, 16, device=DEV).expand(8, 4, 16)
    for bad in (lambda: lb.attention_bwd(q[:4], q, k, k, o, lse), lambda: lb.attention_bwd(q, q, k, k, o, lse[:4]), lambda: lb.attention_bwd(q, q, k, k, o, lse, out=(one, k, k)),
                lambda: lb.attention_bwd(q, q, k, k, o, lse, out=(q, k[:4], k))):
        with pytest.raises(ValueError):
            bad()
    for bad in (lambda: lb.attention(q.half(), k.half(), k.half()), lambda: lb.attention(q, k.bfloat16(), k), lambda: lb.attention(q.cpu(), k.cpu(), k.cpu()),
                lambda: lb.attention_bwd(q, q, k, k, o.to(torch.uint8), lse), lambda: lb.attention_bwd(q.bfloat16(), q, k, k, o, lse)):
        with pytest.raises(TypeError):
            bad()

"""The cache of 4 bits: what is written, bit by bit, against the rule in 64 bits, what is read back, and attention over it against the formula: pages that
end inside anything, tables with holes, lengths from none, new tokens from one, both types, codes; streams and replays; refusals."""
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


def starts(lens):
    return ints(list(np.cumsum([0] + list(lens))))


def a_table(rng, count, need, spare=2):
    """(table [count, need] of pages in no order, number of pages)."""
    pages = count * need + spare
    return rng.permutation(pages)[:count * need].reshape(count, need).astype(np.int32), pages


def filled(rng, pages, KV, page, D):
    """A cache of values of about unit size, as numpy arrays."""
    x = [rng.standard_normal((pages, KV, page, D)).astype(np.float32) * 2.0 ** rng.integers(-1, 2, (pages, KV, page, 1)) for _ in range(2)]
    return ao.fours(x[0]) + ao.fours(x[1])


def on_device(arrays):
    return lb.KVCache(*[torch.from_numpy(a.copy()).to(DEV) for a in arrays])


def values_of(arrays, table, b, n, page):
    """Keys and values [n, KV, D] of sequence b's first n positions in 64 bits; positions that hold nothing are NaN."""
    out = []
    for c, s in ((arrays[0], arrays[1]), (arrays[2], arrays[3])):
        v = np.full((n, c.shape[1], 2 * c.shape[3]), np.nan)
        for p in range(n):
            if p // page < table.shape[1] and 0 <= table[b, p // page] < c.shape[0]:
                v[p] = ao.fours_values(c[table[b, p // page], :, p % page], s[table[b, p // page], :, p % page])
        out.append(v)
    return out


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("lens,before,KV,D,page", [([1], [0], 1, 32, 1), ([1, 1, 1], [0, 15, 63], 8, 128, 16), ([5, 0, 40], [3, 9, 0], 2, 64, 16), ([70, 130], [0, 0], 3, 96, 64),
                                                   ([33], [100], 12, 64, 7), ([300, 1], [0, 299], 2, 128, 128)])
def test_writes_and_reads(lens, before, KV, D, page, dtype):
    rng = np.random.default_rng(sum(lens) + D)
    total = [n + m for n, m in zip(lens, before)]
    table, pages = a_table(rng, len(lens), max(1, -(-max(total) // page)))
    old = filled(rng, pages, KV, page, D)
    cache = on_device(old)
    k, v = (values(rng, (sum(lens), KV, D), dtype) * np.float32(2.0) ** rng.integers(-20, 20, (sum(lens), KV, 1)).astype(np.float32) for _ in range(2))
    k[::3, :, :32] = 0.0                                 # blocks of nothing
    k[1::3, :, ::2] = k[1::3, :, :1]                     # repeated values, at the borders of roundings where they are the largest
    t, s, ln = torch.from_numpy(table).to(DEV), starts(lens), ints(total)
    lb.cache_write(dev(k, dtype), dev(v, dtype), cache, t, s, ln)
    want = [a.copy() for a in old]
    at = 0
    for b, n in enumerate(lens):
        for i in range(n):
            p = before[b] + i
            for x, j in ((k, 0), (v, 2)):
                want[j][table[b, p // page], :, p % page], want[j + 1][table[b, p // page], :, p % page] = ao.fours(x[at])
            at += 1
    for got, w in zip(cache, want):
        assert np.array_equal(got.cpu().numpy(), w)      # everything else is as it was
    for out in ("f32", "bf16"):
        rk, rv = lb.cache_read(cache, t, starts(total), ln, sum(total), out_dtype=DT[out])
        at = 0
        for b, n in enumerate(total):
            for got, w in zip((rk, rv), values_of(want, table, b, n, page)):
                assert got.dtype == DT[out] and np.array_equal(host(got[at:at + n]), w)
            at += n
    nk, nv = lb.cache_read(cache, t, s, ln, sum(lens))   # the newest alone
    at = 0
    for b, n in enumerate(lens):
        whole = values_of(want, table, b, total[b], page)
        assert np.array_equal(host(nk[at:at + n]), whole[0][before[b]:]) and np.array_equal(host(nv[at:at + n]), whole[1][before[b]:])
        at += n


@pytest.mark.gpu
def test_every_border_of_a_rounding():
    """Blocks whose largest element is each border of the power's rule, with every border of a code and its neighbours inside."""
    mids = [0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0]
    inner = [f(np.float32(m)) for m in mids + list(ao.FOURS[1:7]) for f in (lambda x: x, lambda x: np.nextafter(x, np.float32(0)), lambda x: np.nextafter(x, np.float32(9)))][:29]
    tops = [np.float32(t) for t in (6.0, 3.0000002, 4.0, 5.9999995, 5.0)]
    rows = []
    for e in (-99, -20, 0, 31, 125):
        for t in tops:
            rows.append(np.array([t, -t, 0.0] + inner, np.float32) * np.float32(2.0) ** np.float32(e))
    rows.append(np.full(32, 2.0 ** -127, np.float32))    # subnormal numbers count as zero
    rows.append(np.full(32, 3.4e38, np.float32))         # beyond the largest power: saturates
    rows.append(np.array([2.0 ** -110] + [0.0] * 31, np.float32))
    for bad in (np.inf, -np.inf, np.nan):
        rows.append(np.array([1.0, bad] + [2.0] * 30, np.float32))
    x = np.stack(rows)[:, None]
    n = len(x)
    cache = lb.kv_cache(1, n, 1, 32)
    lb.cache_write(dev(x), dev(-x), cache, ints([[0]]), None if n == 1 else ints([0, n]), ints([n]))
    for codes, scales, w in ((cache.k, cache.k_scale, x), (cache.v, cache.v_scale, -x)):
        c, s = ao.fours(w[:, 0])
        assert np.array_equal(scales.cpu().numpy()[0, 0], s) and np.array_equal(codes.cpu().numpy()[0, 0], c)
    k, _ = lb.cache_read(cache, ints([[0]]), ints([0, n]), ints([n]), n, out_dtype=torch.float32)
    assert k[-3:].isnan().all() and k[:-3].isfinite().all()
    assert (k[-6] == 0).all() and (k[-5] == 6 * 2.0 ** 125).all()


@pytest.mark.gpu
def test_arrangements_views_and_holes():
    rng = np.random.default_rng(2)
    B, L, H, KV, D, page = 3, 4, 6, 2, 64, 8
    table, pages = a_table(rng, B, 3)
    t, ln = torch.from_numpy(table).to(DEV), ints([4, 13, 24])
    qkv = dev(values(rng, (B * L, H + 2 * KV, D), "bf16"), "bf16")
    k, v = qkv[:, H:H + KV], qkv[:, H + KV:]
    caches = [lb.kv_cache(pages, page, KV, D) for _ in range(4)]
    lb.cache_write(k, v, caches[0], t, starts([L] * B), ln)
    lb.cache_write(k.unflatten(0, (B, L)), v.unflatten(0, (B, L)), caches[1], t, None, ln)
    for i in range(L):                                   # one by one, as a server does
        lb.cache_write(k.unflatten(0, (B, L))[:, i], v.unflatten(0, (B, L))[:, i], caches[2], t, None, ln - (L - 1 - i))
    lb.cache_write(k.contiguous(), v.contiguous(), caches[3], t.repeat_interleave(2, 1)[:, ::2], starts([L] * B), ln)    # a table that is a view
    for other in caches[1:]:
        assert all(torch.equal(a, b) for a, b in zip(caches[0], other))
    rk, rv = lb.cache_read(caches[0], t, None, ln, B * L)
    d = torch.full_like(qkv, 7.0)
    out = lb.cache_read(caches[0], t, None, ln, B * L, out=(d[:, H:H + KV], d[:, H + KV:]))
    assert torch.equal(out[0], rk) and torch.equal(d[:, H + KV:], rv) and (d[:, :H] == 7).all()
    # lens below the rows that are written, pages that are none, positions behind the table: dropped, and read as zeros
    for holes, short in ((t, [2, 13, 40]), (torch.where(t == t[1, 0], -1, t), [4, 8, 24]), (torch.where(t == t[0, 0], pages, t), [4, 13, 24]), (t[:, :1], [4, 13, 24])):
        before = [c.clone() for c in caches[0]]
        cache = lb.KVCache(*[torch.cat([torch.full_like(c[:1], 0xAA), c, torch.full_like(c[:1], 0xAA)]) for c in caches[0]])
        inner = lb.KVCache(*[c[1:-1] for c in cache])
        lb.cache_write(k, v, inner, holes.contiguous(), starts([L] * B), ints(short))
        assert all((c[0] == 0xAA).all() and (c[-1] == 0xAA).all() for c in cache)
        rk, _ = lb.cache_read(inner, holes, starts([L] * B), ints(short), B * L)
        for b in range(B):
            for i in range(L):
                p = short[b] - L + i
                there = p >= 0 and p // page < holes.shape[1] and 0 <= int(holes[b, p // page]) < pages
                want = ao.fours_values(*ao.fours(host(k[b * L + i]).astype(np.float32))) if there else 0.0
                assert np.array_equal(host(rk[b * L + i]), np.broadcast_to(want, (KV, D)))
        del before
    # rows of no sequence
    s = ints([2, 6, 6, 9])
    k2, v2 = lb.cache_read(caches[0], t, s, ln, B * L)
    assert not k2[:2].any() and not v2[9:].any() and k2[2:9].any()
    held = [torch.full_like(k2, 7.0) for _ in range(2)]
    lb.cache_read(caches[0], t, s, ln, B * L, out=held)
    assert (held[0][:2] == 7).all() and (held[1][9:] == 7).all() and torch.equal(held[0][2:9], k2[2:9])
    empty = lb.cache_read(caches[0], t, ints([0, 0, 0, 0]), ln, 0)
    assert empty[0].shape == (0, KV, D)


def expected(arrays, table, q, lens, page, dtype, scale):
    """(value, bound) of attention of q [sequences, fresh, H, D]."""
    want, tol, fresh, KV = np.zeros(q.shape), np.zeros(q.shape), q.shape[1], arrays[0].shape[1]
    for b, n in enumerate(lens):
        n = max(n, 0)
        k, v = values_of(arrays, table, b, n, page)
        there = ~np.isnan(k[:, 0, 0])
        see = (np.arange(n)[None] <= np.arange(fresh)[:, None] + (lens[b] - fresh)) & there[None]
        for h in range(q.shape[2]):
            kv = h // (q.shape[2] // KV)
            f = ao.attend(q[b, :, h], np.nan_to_num(k[:, kv]), np.nan_to_num(v[:, kv]), see, float(np.float32(scale)), dtype, 1 if dtype == "bf16" else 3)
            want[b, :, h], tol[b, :, h] = f["o"], f["to"]
    return want, tol


def check(lens, fresh, H, KV, D, page, dtype, scale=None, holes=False, room=0):
    rng = np.random.default_rng(sum(lens) + 13 * D + fresh)
    need = max(1, -(-max(lens) // page)) + room
    table, pages = a_table(rng, len(lens), need)
    if holes:
        table[rng.random(table.shape) < 0.4] = -1
        table[0, 0] = pages
    arrays = filled(rng, pages, KV, page, D)
    q = values(rng, (len(lens), fresh, H, D), dtype)
    cache, t, ln = on_device(arrays), torch.from_numpy(table).to(DEV), ints(lens)
    want, tol = expected(arrays, table, q, lens, page, dtype, D ** -0.5 if scale is None else scale)
    tq = dev(q, dtype)
    got = lb.cache_attention(tq, cache, t, ln, scale=scale)
    assert got.dtype == DT[dtype] and got.shape == tq.shape
    near(got, want, tol, dtype)
    return want, tol, (tq, cache, t, ln, got)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("lens,fresh,H,KV,D,page", [
    ([1], 1, 1, 1, 32, 1), ([129], 1, 12, 12, 64, 16), ([1, 2, 15, 16, 17, 31, 33], 1, 8, 2, 128, 16), ([700, 3, 0, 64], 1, 32, 8, 128, 64), ([100, 1000], 1, 6, 1, 96, 7),
    ([40, 300], 5, 4, 2, 64, 32), ([3, 200], 9, 40, 2, 128, 64), ([2050], 1, 16, 1, 128, 128), ([513, 511], 2, 3, 3, 32, 5), ([90, 17], 33, 2, 1, 64, 16), ([600], 1, 64, 2, 64, 1024),
    ([-3, 5], 2, 2, 2, 32, 4)])
def test_attention(lens, fresh, H, KV, D, page, dtype):
    check(lens, fresh, H, KV, D, page, dtype)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_attention_over_long_and_broken_tables(dtype):
    check([9000], 1, 8, 2, 128, 64, dtype)
    check([5000, 1, 333], 3, 4, 2, 64, 16, dtype, room=40)
    check([500, 64, 300], 2, 4, 2, 128, 16, dtype, holes=True)
    check([150, 20], 1, 4, 2, 64, 16, dtype, scale=2.0)
    check([150, 20], 1, 4, 2, 64, 16, dtype, scale=0.0)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_attention_output_types(dtype):
    want, tol, (q, cache, t, ln, got) = check([65, 130, 3], 1, 8, 2, 64, 16, dtype)
    for out in ("f32", "bf16"):
        near(lb.cache_attention(q, cache, t, ln, out_dtype=DT[out]), want, tol, out)
    for fmt in ((4, 3, 7 + 6), (3, 4, 3 + 2), (5, 2, 15)):
        codes = lb.cache_attention(q, cache, t, ln, out_dtype=torch.uint8, out_fmt=fmt)
        lo.check_codes(codes.cpu().numpy(), want, tol + 2 * lo.U * np.abs(want), fmt)
    one = lb.cache_attention(q[:, 0], cache, t, ln)
    assert torch.equal(one, got[:, 0])
    held = torch.empty_like(q)
    assert lb.cache_attention(q, cache, t, ln, out=held) is held and torch.equal(held, got)
    wide = torch.cat([q, q], 2)
    assert torch.equal(lb.cache_attention(wide[:, :, :8], cache, t, ln), got)        # queries inside a product's output


@pytest.mark.gpu
@pytest.mark.parametrize("length,fresh,H,KV,D", [(70, 1, 4, 2, 64), (700, 2, 2, 1, 128), (9, 3, 20, 1, 32), (33, 1, 3, 3, 96), (2100, 1, 2, 2, 128)])
def test_float32_outputs_of_bfloat16_queries(length, fresh, H, KV, D):
    """Weights are not rounded then: the bounds are those of three pieces."""
    g = torch.Generator(device="cuda").manual_seed(length)
    cache, table, lens = lb.kv_cache(length // 16 + 1, 16, KV, D), torch.arange(length // 16 + 1, dtype=torch.int32, device="cuda")[None], torch.tensor([length], dtype=torch.int32).cuda()
    x = torch.randn(2, 1, length, KV, D, device="cuda", generator=g)
    lb.cache_write(x[0], x[1], cache, table, None, lens)
    k, v = lb.cache_read(cache, table, None, lens, length, out_dtype=torch.float32)
    q = torch.randn(1, fresh, H, D, device="cuda", generator=g).bfloat16()
    got = lb.cache_attention(q, cache, table, lens, out_dtype=torch.float32)
    for h in range(H):
        kv = h // (H // KV)
        f = ao.attend(*(t.double().cpu().numpy() for t in (q[0, :, h], k[:, kv], v[:, kv])), ao.seen(fresh, length, True), float(np.float32(D ** -0.5)), "f32", 3)
        near(got[0, :, h], f["o"], f["to"] + 2 * lo.U * np.abs(f["o"]), h)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_what_is_not_seen_does_not_matter(dtype):
    """NaN in the lines behind a sequence's last token, in other pages, and in tokens that a query does not see yet."""
    rng = np.random.default_rng(6)
    page, KV, D, lens, fresh = 16, 2, 64, [50, 5], 3
    table, pages = a_table(rng, 2, 5)
    arrays = filled(rng, pages, KV, page, D)
    q = values(rng, (2, fresh, 4, D), dtype)
    t, ln = torch.from_numpy(table).to(DEV), ints(lens)
    want, tol = expected(arrays, table, q, lens, page, dtype, D ** -0.5)
    keep = np.zeros((pages, page), bool)
    for b, n in enumerate(lens):
        for p in range(n - 1):                           # the last token is for the last query alone
            keep[table[b, p // page], p % page] = True
    for s in (1, 3):
        arrays[s][~np.broadcast_to(keep[:, None], arrays[s].shape[:3])] = 255
    got = lb.cache_attention(dev(q, dtype), on_device(arrays), t, ln)
    near(got[:, :-1], want[:, :-1], tol[:, :-1], dtype)
    assert got[:, -1].isnan().all()


@pytest.mark.gpu
def test_streams_and_replays():
    rng = np.random.default_rng(7)
    B, H, KV, D, page = 3, 8, 2, 128, 16
    table, pages = a_table(rng, B, 20)
    t, ln = torch.from_numpy(table).to(DEV), ints([5, 17, 200])
    cache = on_device(filled(rng, pages, KV, page, D))
    qkv = torch.randn(B, H + 2 * KV, D, device=DEV).bfloat16()
    step = lambda c, s=None: (lb.cache_write(qkv[:, H:H + KV], qkv[:, H + KV:], c, t, None, ln, stream=s), lb.cache_attention(qkv[:, :H], c, t, ln, stream=s))[1]  # noqa: E731
    first = lb.KVCache(*[c.clone() for c in cache])
    want = step(first)
    s = torch.cuda.Stream()
    other = lb.KVCache(*[c.clone() for c in cache])
    s.wait_stream(torch.cuda.current_stream())
    got = step(other, s)
    s.synchronize()
    assert torch.equal(got, want) and all(torch.equal(a, b) for a, b in zip(first, other))
    g, own = torch.cuda.CUDAGraph(), lb.KVCache(*[c.clone() for c in cache])
    with torch.cuda.graph(g):
        out = step(own)
        k, v = lb.cache_read(own, t, None, ln, B)
    eager = lb.KVCache(*[c.clone() for c in cache])
    for c, e in zip(own, cache):
        c.copy_(e)
    for _ in range(30):                                  # a server's loop: each replay adds a token
        qkv.copy_(torch.randn_like(qkv))
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, step(eager)) and all(torch.equal(a, b) for a, b in zip(own, eager))
        ek, ev = lb.cache_read(eager, t, None, ln, B)
        assert torch.equal(k, ek) and torch.equal(v, ev)
        ln.add_(1)


@pytest.mark.gpu
def test_offsets_beyond_32_bits():
    pages, KV, page, D = (1 << 20) + 3, 1, 64, 128       # 4.3 GB of codes
    cache = lb.kv_cache(pages, page, KV, D)
    rng = np.random.default_rng(8)
    k, v, q = (dev(values(rng, (100, 1, D), "bf16"), "bf16") for _ in range(3))
    t, ln = ints([[pages - 1, 5, pages - 3]]), ints([100])
    small = lb.kv_cache(3, page, KV, D)
    for c, table in ((cache, t), (small, ints([[2, 1, 0]]))):
        lb.cache_write(k, v, c, table, ints([0, 100]), ln)
    assert torch.equal(cache.k[pages - 1], small.k[2]) and torch.equal(cache.v[pages - 3], small.v[0])
    for a, b in zip(lb.cache_read(cache, t, ints([0, 100]), ln, 100), lb.cache_read(small, ints([[2, 1, 0]]), ints([0, 100]), ln, 100)):
        assert torch.equal(a, b)
    assert torch.equal(lb.cache_attention(q[None], cache, t, ln), lb.cache_attention(q[None], small, ints([[2, 1, 0]]), ln))


@pytest.mark.gpu
def test_nothing_to_do():
    cache = lb.kv_cache(2, 4, 2, 32)
    t0, l0 = torch.empty((0, 3), dtype=torch.int32, device=DEV), torch.empty(0, dtype=torch.int32, device=DEV)
    e = torch.empty(0, 2, 32, device=DEV)
    lb.cache_write(e, e, cache, t0, None, l0)
    assert lb.cache_attention(torch.empty(0, 4, 32, device=DEV), cache, t0, l0).shape == (0, 4, 32)
    q = torch.randn(2, 4, 32, device=DEV)
    none = torch.empty((2, 0), dtype=torch.int32, device=DEV)
    assert not lb.cache_attention(q, cache, none, ints([5, 5])).any()                # a table of no pages
    assert not lb.cache_attention(q, cache, ints([[0], [1]]), ints([0, -7])).any()
    k, v = lb.cache_read(cache, none, None, ints([5, 5]), 2)
    assert not k.any() and not v.any()


def desc(**k):
    P = 0x1000
    d = dict(k=P, ks=P, v=P, vs=P, pages=4, row=2, count=2, table=P, lens=P, page=16, KV=2, D=64)
    return lb.lba_cache4(*{**d, **k}.values())


@pytest.mark.gpu
def test_tables_with_room_for_more_than_a_launch_has_workgroups():
    """2048 sequences that may have 2^30 positions each: a chunk is then a whole sequence, not 2^31 positions."""
    count, row, page = 2048, 16384, 65536
    cache = lb.kv_cache(1, page, 1, 32)
    table = torch.full((count, row), -1, dtype=torch.int32, device="cuda")
    table[:, 0] = 0
    k, v, q = (torch.randn(1, 5, h, 32, device="cuda") for h in (1, 1, 2))
    lens = torch.full((count,), 5, dtype=torch.int32, device="cuda")
    lb.cache_write(k, v, cache, table[:1], None, lens[:1])
    got = lb.cache_attention(q[:, 4].expand(count, 2, 32), cache, table, lens)
    want = lb.cache_attention(q[:, 4], cache, table[:1, :1], lens[:1])
    assert bool(want.any()) and torch.equal(got, want.expand(count, 2, 32))


@pytest.mark.gpu
def test_rows_of_no_sequences_at_all():
    cache = lb.kv_cache(2, 4, 1, 32)
    none, starts = torch.zeros(0, dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    k, v = lb.cache_read(cache, none.view(0, 3), starts, none, 4)
    assert k.shape == (4, 1, 32) and not k.any() and not v.any()
    q = torch.randn(4, 2, 32, device="cuda")
    o, lse = lb.attention(q, q, q, starts=starts, want_stats=True)
    assert not o.any() and bool((lse == -np.inf).all())
    assert not any(d.any() for d in lb.attention_bwd(q, q, q, q, o, lse, starts=starts))


def test_refusals():
    P, W, f, s = ctypes.c_void_p(0x1000), ctypes.c_void_p(0x2000), (4, 3, 7), lb.lba_strides(128, 64)
    write = lambda c=None, **k: lb.lba_cache_write(*{**dict(c=c or desc(), st=None, T=4, K=P, ka=s, V=P, va=s, t=0), **k}.values())  # noqa: E731
    read = lambda c=None, **k: lb.lba_cache_read(*{**dict(c=c or desc(), st=None, T=4, K=P, ka=s, V=P, va=s, t=0, clear=0), **k}.values())  # noqa: E731
    need = lb.lba_cache_attention_workspace_bytes(2, 2, 16, 1, 4, 2, 64)
    attend = lambda c=None, **k: lb.lba_cache_attention(*{**dict(c=c or desc(), Q=P, qa=s, t=0, fresh=1, H=4, scale=0.1, O=P, ot=0, f=f, ws=W, n=need), **k}.values())  # noqa: E731
    for fn in (write, read, attend):
        for bad in (dict(pages=-1), dict(pages=1 << 31), dict(row=-1), dict(row=1 << 31), dict(count=-1), dict(count=(1 << 20) + 1), dict(page=0), dict(page=65537), dict(KV=-1), dict(KV=65536),
                    dict(D=0), dict(D=48), dict(D=160)):
            assert fn(desc(**bad)) == lb.ERR_SHAPE, bad
        assert fn(desc(lens=None)) == lb.ERR_NULL and fn(desc(table=None)) == lb.ERR_NULL
        for w in ("k", "ks", "v", "vs"):
            assert fn(desc(**{w: None})) == lb.ERR_NULL
        assert fn(t=2) == lb.ERR_UNSUPPORTED
    for fn in (write, read):
        assert fn(T=-1) == lb.ERR_SHAPE and fn(T=5) == lb.ERR_SHAPE and fn(K=None) == lb.ERR_NULL and fn(V=None) == lb.ERR_NULL and fn(ka=lb.lba_strides(-1, 0)) == lb.ERR_SHAPE
        assert fn(T=0, K=None, V=None) == lb.OK
    assert attend(Q=None) == lb.ERR_NULL and attend(O=None) == lb.ERR_NULL and attend(H=3) == lb.ERR_SHAPE and attend(H=65536) == lb.ERR_SHAPE
    assert attend(fresh=-1) == lb.ERR_SHAPE and attend(fresh=1 << 30) == lb.ERR_SHAPE and attend(qa=lb.lba_strides(-1, 0)) == lb.ERR_SHAPE
    assert attend(ot=5) == lb.ERR_UNSUPPORTED and attend(ot=2, f=(1, 6, 0)) == lb.ERR_FORMAT
    assert attend(fresh=0, Q=None) == lb.OK and attend(desc(count=0), Q=None) == lb.OK
    need = lb.lba_cache_attention_workspace_bytes(2, 4096, 16, 1, 4, 2, 64)
    if need:
        big = lambda **k: attend(desc(row=4096), **{**dict(n=need), **k})  # noqa: E731
        assert big(ws=None) == lb.ERR_NULL and big(n=need - 1) == lb.ERR_SHAPE and big(ws=ctypes.c_void_p(0x2040)) == lb.ERR_ALIGN


@pytest.mark.gpu
def test_refusals_of_tensors():
    cache, t, ln = lb.kv_cache(4, 8, 2, 32), ints([[0, 1], [2, 3]]), ints([3, 4])
    k, q = torch.randn(2, 2, 32, device=DEV), torch.randn(2, 4, 32, device=DEV)
    for bad in (lambda: lb.kv_cache(4, 8, 2, 48), lambda: lb.cache_write(k[:, :1], k[:, :1], cache, t, None, ln), lambda: lb.cache_write(k[:1], k[:1], cache, t, None, ln),
                lambda: lb.cache_write(k, k, cache, t, ints([0, 2]), ln), lambda: lb.cache_write(k, k, cache, t.long(), None, ln), lambda: lb.cache_write(k, k, cache, t, None, ln[:1]),
                lambda: lb.cache_write(k, k, cache._replace(v=cache.v[:3]), t, None, ln), lambda: lb.cache_write(k, k, cache._replace(k=cache.k.transpose(0, 1)), t, None, ln),
                lambda: lb.cache_read(cache, t, None, ln, 3), lambda: lb.cache_read(cache, t, ints([0, 2]), ln, 2), lambda: lb.cache_read(cache, t, None, ln, 2, out=(k, k.bfloat16())),
                lambda: lb.cache_attention(q[:1], cache, t, ln), lambda: lb.cache_attention(q[:, :3], cache, t, ln), lambda: lb.cache_attention(q[..., :16], cache, t, ln),
                lambda: lb.cache_attention(q, cache, t, ln, out_dtype=torch.uint8)):
        with pytest.raises(ValueError):
            bad()
    for bad in (lambda: lb.cache_write(k.half(), k.half(), cache, t, None, ln), lambda: lb.cache_read(cache, t, None, ln, 2, out_dtype=torch.float16),
                lambda: lb.cache_attention(q.half(), cache, t, ln), lambda: lb.cache_write(k, k.bfloat16(), cache, t, None, ln)):
        with pytest.raises(TypeError):
            bad()

// lba_attn_bwd.h -- the gradients of attention over packed sequences.
//
// Two passes, each with its sums in registers and no atomics: dQ by 128 queries of a head over the keys that they see, then dK and dV by 128 keys
// over the queries that see them, of all heads of a group.  Either makes the scores and the weights' gradient again (seven products in all, where
// one pass with sums in memory needs five).  In the first a lane pair owns a query, as in the forward pass: dQ^T = K^T . S^T.  In the second
// it owns a key: S = Q . K^T, dV^T = G^T . P, dK^T = Q^T . S; what belongs to a query, lse and rowsum(G * O), which the first pass leaves in
// the workspace, is then per register, and read from LDS.
//
// P and S are rounded to bfloat16 (float32: split into pieces) as factors of the sums' products; scores, weights and S themselves are float32.
// Bound by the matrix cores and the weights beside them.  2 sequences of 4096 causal, 32 heads of 128 on 8: dQ, two waves a SIMD, 385 us (1070 TFLOP/s
// of three products), dK and dV 670 (820 of four): its sums, factors and fragments are 448 registers, so that a wave is alone on its SIMD
// and one block's products have to fill what the other's weights leave.
#ifndef LBA_ATTN_BWD_H_
#define LBA_ATTN_BWD_H_

#include "lba_attn_tile.h"

namespace lba {

constexpr float kLog2e = 1.44269504f;

// rowsum(G * O), which S takes off G . V^T, is the sum of P * (G . V^T) over a query's keys.  Taken from a bfloat16 O it has that rounding, 2^-9 of
// |G . O|, which stays where the difference cancels: few keys, or values with a mean.  So tiles of queries of up to this many steps go over their
// keys before, for the sum itself; the others take O's, if the caller does not ask for the same.  Off, relative to the gradients' norm, with O's and so: two keys 3.8e-3
// and 2.4e-3, 100 keys whose values' mean is their spread 3.5e-3 and 2.3e-3, eight times it 2.1e-2 and 2.4e-3.  Backward passes: 32 sequences of
// 128, 12 heads of 64, 27.7 and 29.7 us, 8 of 512, 16 heads of 64, not causal, 50 and 60, 2 of 4096 causal, 32 heads of 128 on 8, 969 and 973; there
// with all tiles so 1219, for 2.48e-3 and 2.36e-3 (1500 keys of values around zero; 4.1e-3 and 2.4e-3 where their mean is their spread).
constexpr int kFewSteps = 8;

template <typename T, int DP, bool DIRECT>
__global__ __launch_bounds__(256, (sizeof(T) == 2 ? DIRECT || DP <= 96 : DP <= 32) ? 2 : 1) void attn_dq_kernel(AttnParams p) {
    constexpr int KT = kStep<T>, KB = KT / 32, KC = DP / 16, DT = DP / 32;
    __shared__ __attribute__((aligned(16))) uint8_t lds[2][2][kTileBytes<T, DP>];                 // buffers of keys and values
    if ((int)blockIdx.x >= p.units * p.slices) {
        const CodeFmt none = {};
        clear_rows(p.starts, p.T, p.count, blockIdx.x - p.units * p.slices, kClearBlocks, (T*)p.dQ, p.dq.row, p.dq.head, p.H, p.D, (float*)nullptr, none);
        return;
    }
    const int unit = p.slices > 1 ? blockIdx.x % p.units : unit_of(blockIdx.x, p.units), per = p.tiles * p.group, slice = blockIdx.x / p.units;
    const int kv = unit / per, h = kv * p.group + unit % per % p.group;
    const TileOf at = find_tile(p.starts, p.T, p.starts_k, p.Tk, p.count, kTileRows, p.tiles - 1 - unit % per / p.group);
    if (at.b < 0) return;
    const Rows rq = at.mine, rk = at.other;
    const int lane = threadIdx.x & 63, wave = threadIdx.x / 64, half = lane / 32;
    auto limit = [&](int i) { return keys_seen(p, rq, rk, i); };
    const int i0 = at.t * kTileRows + wave * 32, i = i0 + (lane & 31);
    const int lim = limit(i), least = limit(i0), most = i0 < rq.n ? limit(min(i0 + 31, rq.n - 1)) : 0;
    const Slice part = slice_of(steps_of_queries(p, rq, rk, at.t, KT), p.slices, slice);
    const int first = part.first, tiles = part.last, least_all = limit(at.t * kTileRows);
    if (first >= tiles && slice > 0) return;
    const bool there = i < rq.n;
    const int all = steps_of_queries(p, rq, rk, at.t, KT);
    const bool twice = sizeof(T) == 2 && (all <= kFewSteps || p.fine);                           // (also a part of the steps goes over all)

    Loader<T, DP, DIRECT> lk, lv;
    auto start = [&](int kt, int buf) {                  // tile kt is the next
        lk.start((const T*)p.K + (int64_t)(rk.first + kt * KT) * p.k.row + (int64_t)kv * p.k.head, p.k.row, p.D);
        lv.start((const T*)p.V + (int64_t)(rk.first + kt * KT) * p.v.row + (int64_t)kv * p.v.head, p.v.row, p.D);
        lk.load(lds[buf][0], rk.n - kt * KT);
        lv.load(lds[buf][1], rk.n - kt * KT);
    };
    if (tiles > first) start(twice ? 0 : first, 0);
    const int64_t row = (int64_t)(rq.first + i) * p.H + h;
    Frag<T> q[KC], g[KC];
    float delta = 0.0f;
    const float lse = p.lse[there ? row : (int64_t)rq.first * p.H];
    load_frags<T, DP>((const T*)p.G + row * p.D, there, p.D, half, g);
    if (!twice) {
        Frag<T> o[KC];
        load_frags<T, DP>((const T*)p.O + row * p.D, there, p.D, half, o);
        load_frags<T, DP>((const T*)p.Q + (int64_t)(rq.first + i) * p.q.row + (int64_t)h * p.q.head, there, p.D, half, q);
#pragma unroll
        for (int k = 0; k < KC; ++k) delta += dot(g[k], o[k]);
    } else {
        load_frags<T, DP>((const T*)p.Q + (int64_t)(rq.first + i) * p.q.row + (int64_t)h * p.q.head, there, p.D, half, q);
        arrived(g);
    }
    arrived(q);
    const float base = there ? -lse * kLog2e : 0.0f;
    const float c = p.scale * kLog2e;
    // this tile is there, and the one before it has been read
    auto arrive = [&](int buf) {
        lk.put(lds[buf][0]);
        lv.put(lds[buf][1]);
        asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
    };
    // scores and the weights' gradients of block b
    auto products = [&](const uint8_t* tk, const uint8_t* tv, int b, f32x16& s, f32x16& u) {
        Frag<T> ring[2][2];
        auto fetch = [&](int x) {
            ring[x % 2][0] = row_frag<T, DP>(tk, 32 * b + (lane & 31), x, half);
            ring[x % 2][1] = row_frag<T, DP>(tv, 32 * b + (lane & 31), x, half);
        };
        fetch(0);
#pragma unroll
        for (int x = 0; x < KC; ++x) {
            if (x + 1 < KC) fetch(x + 1);
            __builtin_amdgcn_sched_barrier(0);
            s = product(ring[x % 2][0], q[x], s);
            u = product(ring[x % 2][1], g[x], u);
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    if (twice && tiles > first) {                        // delta first, then the tiles again
        for (int kt = 0; kt < all; ++kt) {
            const int k0 = kt * KT, buf = kt & 1;
            arrive(buf);
            if (kt + 1 < all) {
                lk.load(lds[buf ^ 1][0], rk.n - k0 - KT);
                lv.load(lds[buf ^ 1][1], rk.n - k0 - KT);
            } else {
                start(first, buf ^ 1);
            }
            if (k0 >= most) continue;                    // (the barriers above are everybody's)
#pragma unroll
            for (int b = 0; b < KB; ++b) {
                f32x16 s = {}, u = {};
                products(lds[buf][0], lds[buf][1], b, s, u);
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    const float w = __builtin_amdgcn_exp2f(fmaf(s[r], c, base)) * u[r];
                    delta += k0 + 32 * b + row_of(r) + 4 * half >= lim ? 0.0f : w;
                }
            }
        }
    }
    delta = sum_of_halves(delta);
    if (there && half == 0 && slice == 0) p.delta[row] = delta;

    f32x16 acc[DT];
#pragma unroll
    for (int t = 0; t < DT; ++t) acc[t] = f32x16{};
    auto step = [&](int kt, auto edge, int buf) {
        constexpr bool EDGE = decltype(edge)::value != 0;
        const int k0 = kt * KT;
        uint8_t* const tk = lds[buf][0];
        uint8_t* const tv = lds[buf][1];
        arrive(buf);
        if (kt + 1 < tiles) {
            lk.load(lds[buf ^ 1][0], rk.n - k0 - KT);
            lv.load(lds[buf ^ 1][1], rk.n - k0 - KT);
        }
        bool broken = false;
        if constexpr (EDGE) {
            broken = p.causal && k0 + KT > least_all && tile_is_broken<T, DP>(tk);
            if (k0 >= most) return;
        }
#pragma unroll
        for (int b = 0; b < KB; ++b) {
            f32x16 s = {}, u = {};
            products(tk, tv, b, s, u);
#pragma unroll
            for (int r = 0; r < 16; ++r) s[r] = __builtin_amdgcn_exp2f(fmaf(s[r], c, base)) * (u[r] - delta);
            if (EDGE && k0 + KT > least) {
#pragma unroll
                for (int r = 0; r < 16; ++r)
                    if (k0 + 32 * b + row_of(r) + 4 * half >= lim) s[r] = 0.0f;
            }
#pragma unroll
            for (int x = 0; x < 2; ++x) {
                const Frag<T> w = as_frag<T>(s, x);
                // a hidden key's infinity must not meet a zero; one that is seen has made the weight itself NaN
#pragma unroll
                for (int t = 0; t < DT; ++t) {
                    const Frag<T> a = column_frag<T, DP>(tk, 32 * b + 16 * x, t, lane);
                    acc[t] = product(EDGE && broken ? without_broken(a) : a, w, acc[t]);
                }
            }
        }
    };
    const int whole = min(tiles, least_all / KT);
    int kt = first;
    const int turned = twice ? all & 1 : 0;              // the first tile's buffer
    if constexpr (DIRECT) {
        if (turned == 0)
            for (; kt + 1 < whole; kt += 2) {
                step(kt, Known<0>{}, 0);
                step(kt + 1, Known<0>{}, 1);
            }
    }
    for (; kt < tiles; ++kt) step(kt, Known<1>{}, (kt - first + turned) & 1);
    if (!there) return;
    const float scale = lim == 1 ? 0.0f : p.scale;       // the weight of an only key is 1 whatever its score is: no residue of G . V^T - rowsum(G * O)
    if (!part.alone) store_columns(p.part + ((int64_t)slice * p.T * p.H + row) * p.D, acc, scale, p.D, half);
    else store_columns((T*)p.dQ + (int64_t)(rq.first + i) * p.dq.row + (int64_t)h * p.dq.head, acc, scale, p.D, half);
}

template <typename T, int DP, bool DIRECT>
__global__ __launch_bounds__(256, DIRECT && sizeof(T) == 2 && DP <= 64 ? 2 : 1) void attn_dkv_kernel(AttnParams p) {
    constexpr int QT = kStep<T>, QB = QT / 32, KC = DP / 16, DT = DP / 32;
    constexpr bool PIPE = !(DIRECT && sizeof(T) == 2 && DP <= 64);
    __shared__ __attribute__((aligned(16))) uint8_t lds[2][2][kTileBytes<T, DP>];                 // buffers of queries and their outputs' gradients
    __shared__ __attribute__((aligned(16))) float side[2][2][QT];                    // -lse in units of log 2, rowsum(G * O)
    if ((int)blockIdx.x >= p.units * p.slices) {
        const CodeFmt none = {};
        clear_rows(p.starts_k, p.Tk, p.count, blockIdx.x - p.units * p.slices, kClearBlocks, (T*)p.dK, p.dk.row, p.dk.head, p.KV, p.D, (float*)nullptr, none);
        clear_rows(p.starts_k, p.Tk, p.count, blockIdx.x - p.units * p.slices, kClearBlocks, (T*)p.dV, p.dv.row, p.dv.head, p.KV, p.D, (float*)nullptr, none);
        return;
    }
    const int unit = p.slices > 1 ? blockIdx.x % p.units : unit_of(blockIdx.x, p.units), kv = unit / p.tiles, slice = blockIdx.x / p.units;
    const TileOf at = find_tile(p.starts_k, p.Tk, p.starts, p.T, p.count, kTileRows, unit % p.tiles);           // earlier tiles, which more queries see, first
    if (at.b < 0) return;
    const Rows rq = at.other, rk = at.mine;
    const int lane = threadIdx.x & 63, wave = threadIdx.x / 64, half = lane / 32;
    auto first_of = [&](int j) { return first_query(p, rq, rk, j); };
    const int j0 = at.t * kTileRows + wave * 32, j = j0 + (lane & 31);
    const bool there = j < rk.n;
    const int lo = first_of(j), lo_wave = first_of(j0), lo_all = first_of(at.t * kTileRows);
    const int t0 = lo_all / QT, steps_head = steps_of_keys(p, rq, rk, at.t, QT);                // tiles of queries of a head; a step is one of a head of the group
    const Slice part = slice_of(steps_head * p.group, p.slices, slice);
    const int steps = part.last;
    if (part.first >= steps && slice > 0) return;
    // a query that sees one key alone has no gradient of its score: where there is one key, all have; else, causal, this one
    const int lone = p.causal ? rq.n - rk.n : -1;
    const float scale = rk.n == 1 ? 0.0f : p.scale;
    const int masked_all = first_of(at.t * kTileRows + kTileRows - 1);                           // from this query on, all of the workgroup's keys are seen

    Loader<T, DP, DIRECT> lq, lg;
    float side_next = 0.0f;                              // lane t of the first two waves: query t % QT of the step's lse or sum
    bool side_there = false;
    int next_tile = part.first % max(1, steps_head), next_head = part.first / max(1, steps_head);
    bool fresh_head = true;
    auto load = [&](int buf) {                           // the step after those that have been loaded
        const int h = kv * p.group + next_head, q0 = (t0 + next_tile) * QT;
        if (fresh_head) {
            lq.start((const T*)p.Q + (int64_t)(rq.first + q0) * p.q.row + (int64_t)h * p.q.head, p.q.row, p.D);
            lg.start((const T*)p.G + ((int64_t)(rq.first + q0) * p.H + h) * p.D, (int64_t)p.H * p.D, p.D);
        }
        lq.load(lds[buf][0], rq.n - q0);
        lg.load(lds[buf][1], rq.n - q0);
        if (threadIdx.x < 2 * QT) {
            const int i = q0 + (int)threadIdx.x % QT;
            const int64_t row = (int64_t)(rq.first + i) * p.H + h;
            const float* from = (int)threadIdx.x < QT ? p.lse : p.delta;
            side_next = from[i < rq.n ? row : (int64_t)rq.first * p.H];              // (used only where it is put down: nothing waits for it here)
            side_there = i < rq.n;
        }
        fresh_head = ++next_tile == steps_head;
        if (fresh_head) { next_tile = 0; ++next_head; }
    };
    if (steps > part.first) load(0);
    Frag<T> k[KC], v[KC];
    load_frags<T, DP>((const T*)p.K + (int64_t)(rk.first + j) * p.k.row + (int64_t)kv * p.k.head, there, p.D, half, k);
    load_frags<T, DP>((const T*)p.V + (int64_t)(rk.first + j) * p.v.row + (int64_t)kv * p.v.head, there, p.D, half, v);
    arrived(k);
    arrived(v);
    const float c = p.scale * kLog2e;

    f32x16 dk[DT], dv[DT];
#pragma unroll
    for (int t = 0; t < DT; ++t) { dk[t] = f32x16{}; dv[t] = f32x16{}; }
    int n = part.first;                                  // steps that are done
    // One tile of queries.  EDGE: some key may not be seen by all of them.  PIPE: the products of one block of 32 queries run while the weights of the
    // other are worked out, since a wave that is alone on its SIMD has only its own instructions to fill it; else two waves share it.
    auto step = [&](int tile, auto edge) {
        constexpr bool EDGE = decltype(edge)::value != 0;
        const int q0 = (t0 + tile) * QT, buf = (n - part.first) & 1;
        uint8_t* const tq = lds[buf][0];
        uint8_t* const tg = lds[buf][1];
        lq.put(tq);
        lg.put(tg);
        if (threadIdx.x < 2 * QT) {                      // rows that are not there have no weight
            const bool sum = threadIdx.x >= QT;
            side[buf][sum][threadIdx.x % QT] = sum ? (side_there ? side_next : 0.0f) : side_there ? -side_next * kLog2e : -__builtin_inff();
        }
        asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        if (++n < steps) load(buf ^ 1);
        if constexpr (EDGE) {
            // Some key is not seen by all: zeros for infinities and NaN.  A query that has any has them in lse or rowsum(G * O) too, and so as a weight.
            if (p.causal && q0 < masked_all) {
                const bool a = tile_is_broken<T, DP>(tq), b = tile_is_broken<T, DP>(tg);
                if (a) clean_tile<T, DP>(tq);
                if (b) clean_tile<T, DP>(tg);
                if ((a || b) && threadIdx.x < QT && !(fabsf(side[buf][1][threadIdx.x]) < __builtin_inff())) side[buf][0][threadIdx.x] = __builtin_nanf("");
                if (a || b) __syncthreads();
            }
            if (q0 + QT <= lo_wave) return;
        }
        constexpr int RING = sizeof(T) == 2 ? 3 : 2;     // fragments that are under way or in use
        f32x16 s[PIPE ? QB : 1], u[PIPE ? QB : 1];
        Frag<T> w[PIPE ? QB : 1][2], f[PIPE ? QB : 1][2];
        f32x4_t base[4], delta[4];
        auto at = [](int b) { return PIPE ? b : 0; };
        auto sides = [&](int b) {
#pragma unroll
            for (int x = 0; x < 4; ++x) {
                base[x] = *(const f32x4_t*)&side[buf][0][32 * b + 8 * x + 4 * half];
                delta[x] = *(const f32x4_t*)&side[buf][1][32 * b + 8 * x + 4 * half];
            }
        };
        auto weights = [&](int b, int first, int last) { // registers first .. last - 1 of block b
#pragma unroll
            for (int r = first; r < last; ++r) {
                float& x = ((float*)&s[at(b)])[r];
                float& y = ((float*)&u[at(b)])[r];
                x = __builtin_amdgcn_exp2f(fmaf(x, c, base[r / 4][r % 4]));
                y = x * (y - delta[r / 4][r % 4]);
                if (EDGE && q0 + 32 * b + row_of(r) + 4 * half < lo) x = y = 0.0f;
                if (EDGE && q0 + 32 * b + row_of(r) + 4 * half == lone) y = 0.0f;
            }
        };
        auto pack = [&](int b) {
#pragma unroll
            for (int x = 0; x < 2; ++x) { w[at(b)][x] = as_frag<T>(s[at(b)], x); f[at(b)][x] = as_frag<T>(u[at(b)], x); }
        };
        auto scores = [&](int b) {                       // and PIPE the weights of the block before
            Frag<T> ring[RING][2];
            auto fetch = [&](int x) {
                ring[x % RING][0] = row_frag<T, DP>(tq, 32 * b + (lane & 31), x, half);
                ring[x % RING][1] = row_frag<T, DP>(tg, 32 * b + (lane & 31), x, half);
            };
            s[at(b)] = u[at(b)] = f32x16{};
            fetch(0);
            if (RING > 2) fetch(1);
            if (!PIPE) sides(b);
            else if (b > 0) sides(b - 1);
#pragma unroll
            for (int x = 0; x < KC; ++x) {
                if (x + RING - 1 < KC) fetch(x + RING - 1);
                __builtin_amdgcn_sched_barrier(0);
                s[at(b)] = product(ring[x % RING][0], k[x], s[at(b)]);
                u[at(b)] = product(ring[x % RING][1], v[x], u[at(b)]);
                if (PIPE && b > 0) weights(b - 1, 16 * x / KC, 16 * (x + 1) / KC);
                __builtin_amdgcn_sched_barrier(0);
            }
            if (PIPE && b > 0) pack(b - 1);
        };
        auto sums = [&](int b) {                         // and PIPE, with the first block, the weights of the last
            constexpr int N = 2 * DT;                    // column tiles of both halves of the block
            const bool last = PIPE && QB > 1 && b == 0;
            Frag<T> ring[RING][2];
            auto fetch = [&](int i) {
                ring[i % RING][0] = column_frag<T, DP>(tg, 32 * b + 16 * (i / DT), i % DT, lane);
                ring[i % RING][1] = column_frag<T, DP>(tq, 32 * b + 16 * (i / DT), i % DT, lane);
            };
            fetch(0);
            if (RING > 2) fetch(1);
#pragma unroll
            for (int i = 0; i < N; ++i) {
                if (i + RING - 1 < N) fetch(i + RING - 1);
                __builtin_amdgcn_sched_barrier(0);
                dv[i % DT] = product(ring[i % RING][0], w[at(b)][i / DT], dv[i % DT]);
                dk[i % DT] = product(ring[i % RING][1], f[at(b)][i / DT], dk[i % DT]);
                if (last) weights(QB - 1, 16 * i / N, 16 * (i + 1) / N);
                __builtin_amdgcn_sched_barrier(0);
            }
            if (last) pack(QB - 1);
        };
        if constexpr (PIPE && QB > 1) {
#pragma unroll
            for (int b = 0; b < QB; ++b) scores(b);
            sides(QB - 1);
#pragma unroll
            for (int b = 0; b < QB; ++b) sums(b);
        } else {
#pragma unroll
            for (int b = 0; b < QB; ++b) {
                scores(b);
                if (PIPE) sides(b);
                weights(b, 0, 16);
                pack(b);
                sums(b);
            }
        }
    };
    // of every head the steps at the edge, then those that all the workgroup's keys are seen by
    const int edge = max(0, min(steps_head, (masked_all + QT - 1) / QT - t0));
    while (n < steps) {
        const int tile = n % steps_head, head = n - tile;
        for (int last = min(steps, head + edge); n < last;) step(n - head, Known<1>{});
        for (int last = min(steps, head + steps_head); n < last;) step(n - head, Known<0>{});
    }
    if (!there) return;
    if (!part.alone) {
        const int64_t rows = (int64_t)p.Tk * p.KV, to = slice * rows + (int64_t)(rk.first + j) * p.KV + kv;
        store_columns(p.part + to * p.D, dk, scale, p.D, half);
        store_columns(p.part + (p.slices * rows + to) * p.D, dv, 1.0f, p.D, half);
        return;
    }
    store_columns((T*)p.dK + (int64_t)(rk.first + j) * p.dk.row + (int64_t)kv * p.dk.head, dk, scale, p.D, half);
    store_columns((T*)p.dV + (int64_t)(rk.first + j) * p.dv.row + (int64_t)kv * p.dv.head, dv, 1.0f, p.D, half);
}

template <typename T> void launch_attn_dq(const AttnParams& p, bool direct, hipStream_t st) {
    const dim3 grid((unsigned)(p.units * p.slices + (p.clear && p.starts ? kClearBlocks : 0)));
#define LBA_ATTN(DP) \
    if (p.D <= DP) { \
        if (sizeof(T) == 2 && direct) hipLaunchKernelGGL((attn_dq_kernel<T, DP, sizeof(T) == 2>), grid, dim3(256), 0, st, p); \
        else hipLaunchKernelGGL((attn_dq_kernel<T, DP, false>), grid, dim3(256), 0, st, p); \
        return; \
    }
    LBA_ATTN(32)
    LBA_ATTN(64)
    LBA_ATTN(96)
    LBA_ATTN(128)
#undef LBA_ATTN
}
template <typename T> void launch_attn_dkv(const AttnParams& p, bool direct, hipStream_t st) {
    const dim3 grid((unsigned)(p.units * p.slices + (p.clear && p.starts_k ? kClearBlocks : 0)));
#define LBA_ATTN(DP) \
    if (p.D <= DP) { \
        if (sizeof(T) == 2 && direct) hipLaunchKernelGGL((attn_dkv_kernel<T, DP, sizeof(T) == 2>), grid, dim3(256), 0, st, p); \
        else hipLaunchKernelGGL((attn_dkv_kernel<T, DP, false>), grid, dim3(256), 0, st, p); \
        return; \
    }
    LBA_ATTN(32)
    LBA_ATTN(64)
    LBA_ATTN(96)
    LBA_ATTN(128)
#undef LBA_ATTN
}

}  // namespace lba
#endif

// lba_attn_fwd.h -- attention over packed sequences, forward.
//
// A workgroup has 128 queries of a head, a wave 32 of them, one a lane pair; it walks over the keys in tiles of KT, which go to LDS in two buffers. S^T = K . Q^T
// puts a query's scores into its own two lanes, so that the running maximum and sum are a lane's own numbers but for one exchange a tile, and
// P^T goes on to O^T = V^T . P^T without leaving its registers.  The maximum is moved (and the sums multiplied) only where a score is more than 8
// above it in units of log 2: weights are then at most 256 times the final ones, which changes no rounding.
//
// Weights are rounded to bfloat16 for the second product, which is what the matrix cores take; their sum is not.  Float32, outputs of float32, and who
// asks for it: split into pieces.  (13 prompts of 40 to 2048, 32 heads of 128 on 8, to codes of 4 bits of significand: 116 us so and 207 in pieces.  8.2e-3 of
// the codes' norm are neighbours of the nearest code then, but the output is rounded to within 2.66e-2 of its norm either way.)
// Bound by the matrix cores and what stands beside their 32 products of a wave's step (64 keys, heads of 128): a maximum, a multiply-add, an exponential,
// an addition and half a conversion for each of a lane's 32 scores.  Two waves a SIMD take turns: 2 sequences of 4096 causal, 32 heads of 128, 285 us (960
// TFLOP/s), where 8192^3 of a library product reach 1340.  Short sequences are bound by a workgroup's chain of reads: starts, first tiles, stores.
#ifndef LBA_ATTN_FWD_H_
#define LBA_ATTN_FWD_H_

#include "lba_attn_tile.h"

namespace lba {

// a part's maximum, in units of log 2, and sum of weights
__device__ __forceinline__ void store_end(const AttnParams& p, int64_t to, float top, float sum) {
    float* end = p.part + (int64_t)p.slices * p.T * p.H * p.D + to * 2;
    end[0] = top;
    end[1] = sum;
}

// FINE: bfloat16 whose weights are three pieces too.
// Where rows do not go straight to LDS one loop has all tiles: the code of two, read once each by short sequences, costs more than its edge's tests.
template <typename T, int DP, bool DIRECT, bool FINE>
__global__ __launch_bounds__(256, DIRECT || DP <= 96 ? 2 : 1) void attn_kernel(AttnParams p) {
    static_assert(!FINE || sizeof(T) == 2, "float32 has three pieces in any case");
    constexpr int KT = kStep<T>, KB = KT / 32, KC = DP / 16, DT = DP / 32;
    __shared__ __attribute__((aligned(16))) uint8_t lds[2][2][kTileBytes<T, DP>];                 // buffers of keys and values
    __shared__ uint32_t firsts[DP];                      // of a tile whose values hold infinities or NaN: where
    if ((int)blockIdx.x >= p.units * p.slices) {
        with_output(p, [&](auto* o) { clear_rows(p.starts, p.T, p.count, blockIdx.x - p.units * p.slices, kClearBlocks, o, (int64_t)p.H * p.D, p.D, p.H, p.D, p.lse, p.fmt); });
        return;
    }
    const int unit = p.slices > 1 ? blockIdx.x % p.units : unit_of(blockIdx.x, p.units), per = p.tiles * p.group, slice = blockIdx.x / p.units;
    const int kv = unit / per, h = kv * p.group + unit % per % p.group;
    const TileOf at = find_tile(p.starts, p.T, p.starts_k, p.Tk, p.count, kTileRows, p.tiles - 1 - unit % per / p.group);               // later tiles of a sequence, which see more, first
    if (at.b < 0) return;
    const Rows rq = at.mine, rk = at.other;
    const int lane = threadIdx.x & 63, wave = threadIdx.x / 64, half = lane / 32;
    auto limit = [&](int i) { return keys_seen(p, rq, rk, i); };
    const int i0 = at.t * kTileRows + wave * 32, i = i0 + (lane & 31);
    const int lim = limit(i), least = limit(i0), most = i0 < rq.n ? limit(min(i0 + 31, rq.n - 1)) : 0;
    const Slice part = slice_of(steps_of_queries(p, rq, rk, at.t, KT), p.slices, slice);
    const int first = part.first, tiles = part.last, least_all = limit(at.t * kTileRows);
    if (first >= tiles && slice > 0) return;

    Loader<T, DP, DIRECT> lk, lv;
    lk.start((const T*)p.K + (int64_t)(rk.first + first * KT) * p.k.row + (int64_t)kv * p.k.head, p.k.row, p.D);
    lv.start((const T*)p.V + (int64_t)(rk.first + first * KT) * p.v.row + (int64_t)kv * p.v.head, p.v.row, p.D);
    if (tiles > first) {
        lk.load(lds[0][0], rk.n - first * KT);
        lv.load(lds[0][1], rk.n - first * KT);
    }
    Frag<T> q[KC];
    load_frags<T, DP>((const T*)p.Q + (int64_t)(rq.first + i) * p.q.row + (int64_t)h * p.q.head, i < rq.n, p.D, half, q);
    arrived(q);
    float c = p.scale * 1.44269504f;                     // weights are 2^(c s); c > 0 after this
    if (!(c > 0.0f)) {
#pragma unroll
        for (int k = 0; k < KC; ++k) {
            if constexpr (sizeof(T) == 2) {
                q[k].w = c == 0.0f ? i32x4_t{0, 0, 0, 0} : q[k].w ^ (int32_t)0x80008000;
            } else {
#pragma unroll
                for (int n = 0; n < 3; ++n) q[k].w[n] = c == 0.0f ? i32x4_t{0, 0, 0, 0} : q[k].w[n] ^ (int32_t)0x80008000;
            }
        }
        c = c == 0.0f ? 1.0f : -c;
    }

    f32x16 acc[DT];
#pragma unroll
    for (int t = 0; t < DT; ++t) acc[t] = f32x16{};
    float top = -__builtin_inff(), sum = 0.0f;           // of this lane's query: the maximum in use, times c, and this half's sum
    // One tile.  EDGE: some query may not see all of it; the tiles before are seen whole by every query of the workgroup.
    auto step = [&](int kt, auto edge, int buf) {
        constexpr bool EDGE = decltype(edge)::value != 0;
        const int k0 = kt * KT;
        uint8_t* const tk = lds[buf][0];
        uint8_t* const tv = lds[buf][1];
        lk.put(tk);
        lv.put(tv);
        asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
        __builtin_amdgcn_s_barrier();                    // this tile is there, and the one before it has been read
        asm volatile("" ::: "memory");
        if (kt + 1 < tiles) {
            lk.load(lds[buf ^ 1][0], rk.n - k0 - KT);
            lv.load(lds[buf ^ 1][1], rk.n - k0 - KT);
        }
        // Values that hold infinities or NaN, where some query sees this tile in part, or the weights' smaller pieces, zero or negative, would meet them
        // (float32's values are pieces themselves, of which an infinity is the last, that meets the weight's first alone).
        bool broken = false;
        if constexpr (EDGE || FINE) {
            broken = (FINE || (p.causal && k0 + KT > least_all)) && tile_is_broken<T, DP>(tv);
            if (broken) {
                find_broken<T, DP>(tv, firsts);
                clean_tile<T, DP>(tv);
            }
        }
        if (EDGE && k0 >= most) return;                  // (the barriers above are everybody's)
        f32x16 s[KB];
#pragma unroll
        for (int b = 0; b < KB; ++b) s[b] = f32x16{};
        constexpr int RING = sizeof(T) == 2 ? 3 : 2;     // two steps' rows (float32, of three pieces: one's) are on their way while those before are multiplied
        Frag<T> f[RING][KB];
        auto fetch = [&](int k) {
#pragma unroll
            for (int b = 0; b < KB; ++b) f[k % RING][b] = row_frag<T, DP>(tk, 32 * b + (lane & 31), k, half);
        };
        fetch(0);
        if (RING > 2) fetch(1);
#pragma unroll
        for (int k = 0; k < KC; ++k) {
            if (k + RING - 1 < KC) fetch(k + RING - 1);
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int b = 0; b < KB; ++b) s[b] = product(f[k % RING][b], q[k], s[b]);
            __builtin_amdgcn_sched_barrier(0);
        }
        if (EDGE && k0 + KT > least) {
#pragma unroll
            for (int b = 0; b < KB; ++b)
#pragma unroll
                for (int r = 0; r < 16; ++r)
                    if (k0 + 32 * b + row_of(r) + 4 * half >= lim) s[b][r] = -__builtin_inff();
        }
        float mx = s[0][0];
#pragma unroll
        for (int b = 0; b < KB; ++b)
#pragma unroll
            for (int r = 0; r < 16; ++r) mx = fmaxf(mx, s[b][r]);
        mx = max_of_halves(mx) * c;
        if (__any(mx > top + 8.0f)) {
            const float now = fmaxf(mx, top);
            const float f = now == -__builtin_inff() ? 1.0f : __builtin_amdgcn_exp2f(top - now);
            top = now;
            sum *= f;
#pragma unroll
            for (int t = 0; t < DT; ++t) acc[t] *= f;
        }
        const float base = top == -__builtin_inff() ? 0.0f : -top;
#pragma unroll
        for (int b = 0; b < KB; ++b)
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                s[b][r] = __builtin_amdgcn_exp2f(fmaf(s[b][r], c, base));
                sum += s[b][r];
            }
#pragma unroll
        for (int b = 0; b < KB; ++b)
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                if constexpr (sizeof(T) == 2) {
                    Frag<bf16_t> w[FINE ? 3 : 1];
                    as_factors(s[b], k, w);
#pragma unroll
                    for (int t = 0; t < DT; ++t) {
                        const Frag<bf16_t> x = column_frag<bf16_t, DP>(tv, 32 * b + 16 * k, t, lane);
#pragma unroll
                        for (int n = FINE ? 2 : 0; n >= 0; --n) acc[t] = product(x, w[n], acc[t]);
                    }
                } else {
                    const Frag<T> w = as_frag<T>(s[b], k);
#pragma unroll
                    for (int t = 0; t < DT; ++t) acc[t] = product(column_frag<T, DP>(tv, 32 * b + 16 * k, t, lane), w, acc[t]);
                }
            }
        if constexpr (EDGE || FINE) {
            if (broken) {
                const uint32_t rows = min(max(lim - k0, 0), KT);
#pragma unroll
                for (int t = 0; t < DT; ++t)
#pragma unroll
                    for (int r = 0; r < 16; ++r) acc[t][r] += broken_sum(firsts[32 * t + row_of(r) + 4 * half], rows);
            }
        }
    };
    const int whole = min(tiles, least_all / KT);
    int kt = first;
    if constexpr (DIRECT) {
        for (; kt + 1 < whole; kt += 2) {
            step(kt, Known<0>{}, 0);
            step(kt + 1, Known<0>{}, 1);
        }
    }
    for (; kt < tiles; ++kt) step(kt, Known<1>{}, (kt - first) & 1);
    sum = sum_of_halves(sum);
    if (i >= rq.n) return;
    const int64_t row = (int64_t)(rq.first + i) * p.H + h;
    if (!part.alone) {
        const int64_t rows = (int64_t)p.T * p.H, to = slice * rows + row;
        store_columns(p.part + to * p.D, acc, 1.0f, p.D, half);
        if (half == 0) store_end(p, to, top, sum);
        return;
    }
    const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
    if (p.lse && half == 0) p.lse[row] = sum == 0.0f ? -__builtin_inff() : (top + __builtin_amdgcn_logf(sum)) * 0.693147181f;
    with_output(p, [&](auto* o) {
#pragma unroll
        for (int t = 0; t < DT; ++t)
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                const int d = 32 * t + 8 * g + 4 * half;
                const float v[4] = {acc[t][4 * g] * inv, acc[t][4 * g + 1] * inv, acc[t][4 * g + 2] * inv, acc[t][4 * g + 3] * inv};
                if (d < p.D) store_some<4>(o + row * p.D + d, p.D - d, v, p.fmt);
            }
    });
}

template <typename T> void launch_attn(const AttnParams& p, bool direct, hipStream_t st) {
    constexpr bool BF = sizeof(T) == 2;
    const bool fine = BF && p.fine;
    const dim3 grid((unsigned)(p.units * p.slices + (p.clear && p.starts ? kClearBlocks : 0)));
#define LBA_ATTN(DP) \
    if (p.D <= DP) { \
        if (fine && direct) hipLaunchKernelGGL((attn_kernel<T, DP, BF, BF>), grid, dim3(256), 0, st, p); \
        else if (fine) hipLaunchKernelGGL((attn_kernel<T, DP, false, BF>), grid, dim3(256), 0, st, p); \
        else if (BF && direct) hipLaunchKernelGGL((attn_kernel<T, DP, BF, false>), grid, dim3(256), 0, st, p); \
        else hipLaunchKernelGGL((attn_kernel<T, DP, false, false>), grid, dim3(256), 0, st, p); \
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

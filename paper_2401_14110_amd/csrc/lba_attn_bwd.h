// lba_attn_bwd.h -- the gradients of attention over packed sequences.
//
// Two passes, each with its sums in registers and no atomics: dQ by 128 queries of a head over the keys that they see, then dK and dV by 128 keys
// over the queries that see them, of all heads of a group.  Either makes the scores and the weights' gradient again (seven products in all, where
// one pass with sums in memory needs five).  In the first a lane pair owns a query, as in the forward pass: dQ^T = K^T . S^T.  In the second
// it owns a key: S = Q . K^T, dV^T = G^T . P, dK^T = Q^T . S; what belongs to a query, lse and rowsum(G * O), which the first pass leaves in
// the workspace, is then per register, and read from LDS.
#ifndef LBA_ATTN_BWD_H_
#define LBA_ATTN_BWD_H_

#include "lba_attn_tile.h"

namespace lba {

constexpr float kLog2e = 1.44269504f;

// registers 4 g .. 4 g + 3 of column tiles, times f, to a row
template <typename T, int DT> __device__ __forceinline__ void store_columns(T* row, const f32x16 (&acc)[DT], float f, int D, int half) {
    const CodeFmt none = {};
#pragma unroll
    for (int t = 0; t < DT; ++t)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            const int d = 32 * t + 8 * g + 4 * half;
            const float v[4] = {acc[t][4 * g] * f, acc[t][4 * g + 1] * f, acc[t][4 * g + 2] * f, acc[t][4 * g + 3] * f};
            if (d < D) store_some<4>(row + d, D - d, v, none);
        }
}

// acc += w * (row j of the tile), the columns of this lane's registers: for tiles that hold infinities
template <typename T, int DP, int DT> __device__ __forceinline__ void add_row(f32x16 (&acc)[DT], float w, const uint8_t* tile, int j, int half) {
#pragma unroll
    for (int t = 0; t < DT; ++t)
#pragma unroll
        for (int r = 0; r < 16; ++r) acc[t][r] = fmaf(w, tile_at<T, DP>(tile, j, 32 * t + row_of(r) + 4 * half), acc[t][r]);
}
// the value that row j of a block of 32 has in this lane's column
__device__ __forceinline__ float value_of_row(const f32x16& s, int j, int lane) {
    float w = 0.0f;
#pragma unroll
    for (int r = 0; r < 16; ++r)
        if (row_of(r) == (j & ~4)) w = s[r];
    return __shfl(w, (lane & 31) + 8 * (j & 4));
}

template <typename T, int DP, bool DIRECT>
__global__ __launch_bounds__(256, DIRECT && sizeof(T) == 2 ? 2 : 1) void attn_dq_kernel(AttnParams p) {
    constexpr int KT = sizeof(T) == 2 ? 64 : 32, KB = KT / 32, KC = DP / 16, DT = DP / 32;
    constexpr int TILE = KT * DP * (int)sizeof(T);
    __shared__ __attribute__((aligned(16))) uint8_t lds[2][2][TILE];                 // buffers of keys and values
    if ((int)blockIdx.x >= p.units) {
        const CodeFmt none = {};
        clear_rows(p.starts, p.T, p.count, blockIdx.x - p.units, kClearBlocks, (T*)p.dQ, p.dq.row, p.dq.head, p.H, p.D, (float*)nullptr, none);
        return;
    }
    const int unit = unit_of(blockIdx.x, p.units), per = p.tiles * p.group;
    const int kv = unit / per, h = kv * p.group + unit % per % p.group;
    const TileOf at = find_tile(p.starts, p.T, p.count, kTileRows, p.tiles - 1 - unit % per / p.group);
    if (at.b < 0) return;
    const Rows rq = rows_of(p.starts, p.T, p.count, at.b), rk = rows_of(p.starts_k, p.Tk, p.count, at.b);
    const int lane = threadIdx.x & 63, wave = threadIdx.x / 64, half = lane / 32;
    const int ahead = rk.n - rq.n;
    auto limit = [&](int i) { return p.causal ? max(0, min(rk.n, i + ahead + 1)) : rk.n; };
    const int i0 = at.t * kTileRows + wave * 32, i = i0 + (lane & 31);
    const int lim = limit(i), least = limit(i0), most = i0 < rq.n ? limit(min(i0 + 31, rq.n - 1)) : 0;
    const int tiles = (limit(min(at.t * kTileRows + kTileRows, rq.n) - 1) + KT - 1) / KT, least_all = limit(at.t * kTileRows);
    const bool there = i < rq.n;

    Loader<T, DP, KT, DIRECT> lk, lv;
    lk.start((const T*)p.K + (int64_t)rk.first * p.k.row + (int64_t)kv * p.k.head, p.k.row, p.D);
    lv.start((const T*)p.V + (int64_t)rk.first * p.v.row + (int64_t)kv * p.v.head, p.v.row, p.D);
    if (tiles > 0) {
        lk.load(lds[0][0], rk.n);
        lv.load(lds[0][1], rk.n);
    }
    const int64_t row = (int64_t)(rq.first + i) * p.H + h;
    Frag<T> q[KC], g[KC];
    float delta = 0.0f;
    load_frags<T, DP>((const T*)p.G + row * p.D, there, p.D, half, g);
    load_frags<T, DP>((const T*)p.O + row * p.D, there, p.D, half, q);
#pragma unroll
    for (int k = 0; k < KC; ++k) delta += dot(g[k], q[k]);
    delta = sum_of_halves(delta);
    if (there && half == 0) p.delta[row] = delta;
    const float base = there ? -p.lse[row] * kLog2e : 0.0f;
    load_frags<T, DP>((const T*)p.Q + (int64_t)(rq.first + i) * p.q.row + (int64_t)h * p.q.head, there, p.D, half, q);
    const float c = p.scale * kLog2e;

    f32x16 acc[DT];
#pragma unroll
    for (int t = 0; t < DT; ++t) acc[t] = f32x16{};
    for (int kt = 0; kt < tiles; ++kt) {
        const int k0 = kt * KT;
        uint8_t* const tk = lds[kt & 1][0];
        uint8_t* const tv = lds[kt & 1][1];
        lk.put(tk);
        lv.put(tv);
        asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        if (kt + 1 < tiles) {
            lk.load(lds[(kt + 1) & 1][0], rk.n - k0 - KT);
            lv.load(lds[(kt + 1) & 1][1], rk.n - k0 - KT);
        }
        const bool broken = p.causal && k0 + KT > least_all && tile_is_broken<T, DP, KT>(tk);
        if (k0 >= most) continue;
        const bool masked = k0 + KT > least;
#pragma unroll
        for (int b = 0; b < KB; ++b) {
            f32x16 s = {}, u = {};
#pragma unroll
            for (int k = 0; k < KC; ++k) {
                s = product(row_frag<T, DP>(tk, 32 * b + (lane & 31), k, half), q[k], s);
                u = product(row_frag<T, DP>(tv, 32 * b + (lane & 31), k, half), g[k], u);
            }
#pragma unroll
            for (int r = 0; r < 16; ++r) s[r] = __builtin_amdgcn_exp2f(fmaf(s[r], c, base)) * (u[r] - delta);
            if (masked) {
#pragma unroll
                for (int r = 0; r < 16; ++r)
                    if (k0 + 32 * b + row_of(r) + 4 * half >= lim) s[r] = 0.0f;
            }
            if (!broken) {
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    const Frag<T> w = as_frag<T>(s, k);
#pragma unroll
                    for (int t = 0; t < DT; ++t) acc[t] = product(column_frag<T, DP>(tk, 32 * b + 16 * k, t, lane), w, acc[t]);
                }
            } else {                                     // a hidden key's infinity must not meet a zero: key by key, where it is seen
                for (int j = 0; j < 32 && k0 + 32 * b + j < rk.n; ++j) {
                    const float w = value_of_row(s, j, lane);
                    if (k0 + 32 * b + j < lim) add_row<T, DP>(acc, w, tk, 32 * b + j, half);
                }
            }
        }
    }
    if (there) store_columns((T*)p.dQ + (int64_t)(rq.first + i) * p.dq.row + (int64_t)h * p.dq.head, acc, p.scale, p.D, half);
}

template <typename T, int DP, bool DIRECT>
__global__ __launch_bounds__(256, DIRECT && sizeof(T) == 2 && DP <= 64 ? 2 : 1) void attn_dkv_kernel(AttnParams p) {
    constexpr int QT = sizeof(T) == 2 ? 64 : 32, QB = QT / 32, KC = DP / 16, DT = DP / 32;
    constexpr int TILE = QT * DP * (int)sizeof(T);
    __shared__ __attribute__((aligned(16))) uint8_t lds[2][2][TILE];                 // buffers of queries and their outputs' gradients
    __shared__ __attribute__((aligned(16))) float side[2][2][QT];                    // -lse in units of log 2, rowsum(G * O)
    if ((int)blockIdx.x >= p.units) {
        const CodeFmt none = {};
        clear_rows(p.starts_k, p.Tk, p.count, blockIdx.x - p.units, kClearBlocks, (T*)p.dK, p.dk.row, p.dk.head, p.KV, p.D, (float*)nullptr, none);
        clear_rows(p.starts_k, p.Tk, p.count, blockIdx.x - p.units, kClearBlocks, (T*)p.dV, p.dv.row, p.dv.head, p.KV, p.D, (float*)nullptr, none);
        return;
    }
    const int unit = unit_of(blockIdx.x, p.units), kv = unit / p.tiles;
    const TileOf at = find_tile(p.starts_k, p.Tk, p.count, kTileRows, unit % p.tiles);           // earlier tiles, which more queries see, first
    if (at.b < 0) return;
    const Rows rq = rows_of(p.starts, p.T, p.count, at.b), rk = rows_of(p.starts_k, p.Tk, p.count, at.b);
    const int lane = threadIdx.x & 63, wave = threadIdx.x / 64, half = lane / 32;
    const int ahead = rk.n - rq.n;
    auto first_of = [&](int j) { return p.causal ? max(0, j - ahead) : 0; };                     // the first query that sees key j
    const int j0 = at.t * kTileRows + wave * 32, j = j0 + (lane & 31);
    const bool there = j < rk.n;
    const int lo = first_of(j), lo_wave = first_of(j0), lo_last = first_of(j0 + 31), lo_all = first_of(at.t * kTileRows);
    const int t0 = lo_all / QT, steps_head = rq.n > lo_all ? (rq.n + QT - 1) / QT - t0 : 0, steps = steps_head * p.group;
    const int masked_all = p.causal ? first_of(at.t * kTileRows + kTileRows - 1) : 0;            // from this query on, all of the workgroup's keys are seen

    Loader<T, DP, QT, DIRECT> lq, lg;
    float side_next = 0.0f;                              // lane t of the first two waves: query t % QT of the step's lse or sum
    int next_tile = 0, next_head = 0;
    auto load = [&](int buf) {                           // the step after those that have been loaded
        const int h = kv * p.group + next_head, q0 = (t0 + next_tile) * QT;
        if (next_tile == 0) {
            lq.start((const T*)p.Q + (int64_t)(rq.first + q0) * p.q.row + (int64_t)h * p.q.head, p.q.row, p.D);
            lg.start((const T*)p.G + ((int64_t)(rq.first + q0) * p.H + h) * p.D, (int64_t)p.H * p.D, p.D);
        }
        lq.load(lds[buf][0], rq.n - q0);
        lg.load(lds[buf][1], rq.n - q0);
        if (threadIdx.x < 2 * QT) {
            const int i = q0 + (int)threadIdx.x % QT;
            const int64_t row = (int64_t)(rq.first + i) * p.H + h;
            if ((int)threadIdx.x < QT) side_next = i < rq.n ? -p.lse[row] * kLog2e : -__builtin_inff();              // rows that are not there have no weight
            else side_next = i < rq.n ? p.delta[row] : 0.0f;
        }
        if (++next_tile == steps_head) { next_tile = 0; ++next_head; }
    };
    if (steps > 0) load(0);
    Frag<T> k[KC], v[KC];
    load_frags<T, DP>((const T*)p.K + (int64_t)(rk.first + j) * p.k.row + (int64_t)kv * p.k.head, there, p.D, half, k);
    load_frags<T, DP>((const T*)p.V + (int64_t)(rk.first + j) * p.v.row + (int64_t)kv * p.v.head, there, p.D, half, v);
    const float c = p.scale * kLog2e;

    f32x16 dk[DT], dv[DT];
#pragma unroll
    for (int t = 0; t < DT; ++t) { dk[t] = f32x16{}; dv[t] = f32x16{}; }
    int tile = 0;
    for (int step = 0; step < steps; ++step) {
        const int q0 = (t0 + tile) * QT;
        if (++tile == steps_head) tile = 0;
        uint8_t* const tq = lds[step & 1][0];
        uint8_t* const tg = lds[step & 1][1];
        lq.put(tq);
        lg.put(tg);
        if (threadIdx.x < 2 * QT) side[step & 1][threadIdx.x / QT][threadIdx.x % QT] = side_next;
        asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        if (step + 1 < steps) load((step + 1) & 1);
        bool broken = p.causal && q0 < masked_all;
        if (broken) {
            const bool a = tile_is_broken<T, DP, QT>(tq);
            broken = tile_is_broken<T, DP, QT>(tg) || a;
        }
        if (q0 + QT <= lo_wave) continue;
        const bool masked = q0 < lo_last;
#pragma unroll
        for (int b = 0; b < QB; ++b) {
            f32x16 s = {}, u = {};
#pragma unroll
            for (int x = 0; x < KC; ++x) {
                s = product(row_frag<T, DP>(tq, 32 * b + (lane & 31), x, half), k[x], s);
                u = product(row_frag<T, DP>(tg, 32 * b + (lane & 31), x, half), v[x], u);
            }
#pragma unroll
            for (int x = 0; x < 4; ++x) {
                const f32x4_t base = *(const f32x4_t*)&side[step & 1][0][32 * b + 8 * x + 4 * half];
                const f32x4_t delta = *(const f32x4_t*)&side[step & 1][1][32 * b + 8 * x + 4 * half];
#pragma unroll
                for (int y = 0; y < 4; ++y) {
                    s[4 * x + y] = __builtin_amdgcn_exp2f(fmaf(s[4 * x + y], c, base[y]));
                    u[4 * x + y] = s[4 * x + y] * (u[4 * x + y] - delta[y]);
                }
            }
            if (masked) {
#pragma unroll
                for (int r = 0; r < 16; ++r)
                    if (q0 + 32 * b + row_of(r) + 4 * half < lo) s[r] = u[r] = 0.0f;
            }
            if (!broken) {
#pragma unroll
                for (int x = 0; x < 2; ++x) {
                    const Frag<T> w = as_frag<T>(s, x), f = as_frag<T>(u, x);
#pragma unroll
                    for (int t = 0; t < DT; ++t) {
                        dv[t] = product(column_frag<T, DP>(tg, 32 * b + 16 * x, t, lane), w, dv[t]);
                        dk[t] = product(column_frag<T, DP>(tq, 32 * b + 16 * x, t, lane), f, dk[t]);
                    }
                }
            } else {
                for (int i = 0; i < 32 && q0 + 32 * b + i < rq.n; ++i) {
                    const float w = value_of_row(s, i, lane), f = value_of_row(u, i, lane);
                    if (q0 + 32 * b + i >= lo) {
                        add_row<T, DP>(dv, w, tg, 32 * b + i, half);
                        add_row<T, DP>(dk, f, tq, 32 * b + i, half);
                    }
                }
            }
        }
    }
    if (!there) return;
    store_columns((T*)p.dK + (int64_t)(rk.first + j) * p.dk.row + (int64_t)kv * p.dk.head, dk, p.scale, p.D, half);
    store_columns((T*)p.dV + (int64_t)(rk.first + j) * p.dv.row + (int64_t)kv * p.dv.head, dv, 1.0f, p.D, half);
}

template <typename T> void launch_attn_dq(const AttnParams& p, bool direct, hipStream_t st) {
    const dim3 grid((unsigned)(p.units + (p.clear && p.starts ? kClearBlocks : 0)));
#define LBA_ATTN(DP) \
    if (p.D <= DP) { \
        if (direct) hipLaunchKernelGGL((attn_dq_kernel<T, DP, true>), grid, dim3(256), 0, st, p); \
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
    const dim3 grid((unsigned)(p.units + (p.clear && p.starts_k ? kClearBlocks : 0)));
#define LBA_ATTN(DP) \
    if (p.D <= DP) { \
        if (direct) hipLaunchKernelGGL((attn_dkv_kernel<T, DP, true>), grid, dim3(256), 0, st, p); \
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

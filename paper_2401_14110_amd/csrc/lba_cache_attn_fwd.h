// lba_cache_attn_fwd.h -- attention of new tokens over a cache of 4 bits an element.
//
// A token reads its whole cache, so this is a pass over codes.  A workgroup takes one head of keys of one sequence, up to 16 R rows (the new tokens'
// query heads that share it) and a chunk of positions; its four waves take steps of 32 positions in turn, each with a softmax of its own,
// and meet in LDS at the end.  Chunks leave their sums, maximum and rows in the workspace, where a second launch joins them, always in the
// same order.
// In a step lane l has position l % 16 (and that + 16), elements D / 4 * (l / 16) ..: codes come as they are packed, 8 D bytes a load of the wave (1024
// with heads of 128), and become bfloat16 in registers, which holds a code times a power of two exactly.  S^T = K . Q^T on 16 x 16 x 32 leaves a row's
// scores in four lanes; their weights are the other factor of O^T = V^T . P^T without moving, and V, whose rows have to become columns, goes through
// 32 rows of LDS that are the wave's own: no barriers.  Bound by reading the codes: one sequence of 131071, 8 heads of 128 (143 MB), 31 us, 4.5 TB/s; 64
// of 1000 to 8000 (233 MB) 58 us, 4.0 TB/s, of which the longest chunk, where others have ended, is a part.  Weights are rounded to bfloat16 for
// the product with the values; queries of float32, and weights of them, of outputs of float32, or where the caller asks, are split into three
// bfloat16 pieces, so that products are exact (the 64 sequences 73 us for 60 with an output of float32, 89 in float32).
#ifndef LBA_CACHE_ATTN_FWD_H_
#define LBA_CACHE_ATTN_FWD_H_

#include "lba_cache_attn.h"

namespace lba {

typedef int32_t i32x4_c __attribute__((ext_vector_type(4)));
typedef int16_t i16x4_c __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8_c __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2_c __attribute__((ext_vector_type(2)));

__device__ __forceinline__ float max_of_quarters(float v) {
    const auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
    const auto b = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}
__device__ __forceinline__ float sum_of_quarters(float v) {
    const auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = __uint_as_float(a[0]) + __uint_as_float(a[1]);
    const auto b = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __uint_as_float(b[0]) + __uint_as_float(b[1]);
}

// A number in N bfloat16 pieces.  Not FINITE: an infinity or a NaN is the last, with zeros before it, and pieces before the last stay within bfloat16, so that
// numbers that would round up to infinity do not get one.
template <bool FINITE, int N> __device__ __forceinline__ void split(float x, bf16_t (&piece)[N]) {
    constexpr float TOP = 3.38953139e38f;                // bfloat16's largest number
    const bool is = FINITE || fabsf(x) < __builtin_inff();
#pragma unroll
    for (int i = 0; i < N; ++i) {
        piece[i] = (bf16_t)(FINITE || i == N - 1 ? x : is ? __builtin_amdgcn_fmed3f(x, -TOP, TOP) : 0.0f);
        x -= (float)piece[i];
    }
}

__device__ __forceinline__ f32x4_c product16(const i32x4_c& a, const i32x4_c& b, f32x4_c c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_c, a), __builtin_bit_cast(bf16x8_c, b), c, 0, 0, 0);
}
__device__ __forceinline__ i32x4_c eight_fours(uint32_t w, float scale) {
    return i32x4_c{__builtin_bit_cast(int32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 0)), __builtin_bit_cast(int32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 1)),
                   __builtin_bit_cast(int32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 2)), __builtin_bit_cast(int32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 3))};
}

// A lane's part of a position: D / 4 codes, and the powers of the blocks they are in
template <int D> struct Part {
    static constexpr int KC = D / 32, NS = D == 96 ? 3 : 1;                          // words of codes; blocks that differ between them
    uint32_t w[KC];
    uint8_t e[NS];
    __device__ __forceinline__ void load(const uint8_t* codes, const uint8_t* scales, bool there, uint64_t at, int quarter) {         // at: of the position, in codes
        if (!there) {
#pragma unroll
            for (int i = 0; i < KC; ++i) w[i] = 0;
#pragma unroll
            for (int i = 0; i < NS; ++i) e[i] = 127;
            return;
        }
        typedef typename Vec<uint32_t, KC>::type V;
        typedef V AnyV __attribute__((aligned(1)));
        const V x = *(const AnyV*)(codes + at + quarter * (D / 8));
        if constexpr (KC == 1) {
            w[0] = x;
        } else {
#pragma unroll
            for (int i = 0; i < KC; ++i) w[i] = x[i];
        }
#pragma unroll
        for (int i = 0; i < NS; ++i) e[i] = scales[(at >> 4) + (quarter * (D / 4) + 8 * i) / 32];
    }
    // word i as bfloat16 numbers
    __device__ __forceinline__ i32x4_c values(int i) const {
        const uint32_t s = e[NS == 1 ? 0 : i];
        return eight_fours(s == 0 ? 0u : w[i], __uint_as_float(s << 23));            // the conversion reads an exponent of all ones as NaN
    }
    __device__ __forceinline__ bool broken() const {     // NaN, or codes that may be beyond the numbers
        bool bad = false;
#pragma unroll
        for (int i = 0; i < NS; ++i) bad |= e[i] >= 253;
        return bad;
    }
};

// Rows of values in LDS: piece c of 16 bytes stands at c ^ this, so that 16 rows of one piece, and eight rows of two, meet different banks.
template <int D> __device__ __forceinline__ int value_turn(int r) {
    if constexpr (D == 128) return 2 * (r & 7) + ((r >> 3) & 1);
    else if constexpr (D == 64) return 2 * ((r >> 1) & 3) + ((r >> 3) & 1);
    else return 2 * ((r >> 2) & 1) + ((r >> 3) & 1);
}

__device__ __forceinline__ void lds_words_done() {
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_wave_barrier();
}
// A step's 32 rows of values in the wave's LDS, which hold infinities or NaN: of each column the first row with infinity, with its negative and with NaN, a
// byte each (64: there is none), goes to firsts, since a query sees the first rows; then zeros stand for them.
template <int D> __device__ __forceinline__ void clean_values(uint8_t* values, uint32_t* firsts) {
    const int lane = threadIdx.x & 63;
    lds_words_done();
#pragma clang loop unroll(disable)
    for (int d = lane; d < D; d += 64) {
        uint32_t plus = 64, minus = 64, none = 64;
#pragma clang loop unroll(disable)
        for (int r = 31; r >= 0; --r) {
            const uint32_t e = *(const uint16_t*)(values + r * (D * 2) + ((d / 8) ^ value_turn<D>(r)) * 16 + d % 8 * 2);
            if (e == 0x7F80u) plus = r;
            if (e == 0xFF80u) minus = r;
            if ((e & 0x7FFFu) > 0x7F80u) none = r;
        }
        firsts[d] = plus | minus << 8 | none << 16;
    }
    lds_words_done();
#pragma clang loop unroll(disable)
    for (int i = lane; i < 4 * D; i += 64) {
        i32x4_c x = *(const i32x4_c*)(values + i * 16);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const uint32_t e = (uint32_t)x[j];
            x[j] &= (int32_t)~(((e & 0x7F80u) == 0x7F80u ? 0xFFFFu : 0u) | ((e & 0x7F800000u) == 0x7F800000u ? 0xFFFF0000u : 0u));
        }
        *(i32x4_c*)(values + i * 16) = x;
    }
    lds_words_done();
}
// what a column gets from its infinities and NaN in the `seen` rows that are seen
__device__ __forceinline__ float broken_sum(uint32_t firsts, uint32_t seen) {
    const bool plus = (firsts & 255) < seen, minus = ((firsts >> 8) & 255) < seen, none = firsts >> 16 < seen;
    return none || (plus && minus) ? __builtin_nanf("") : plus ? __builtin_inff() : minus ? -__builtin_inff() : 0.0f;
}

// NW: pieces of the weights.
template <typename T, int D, int R, int NW>
__global__ __launch_bounds__(256, R == 1 && NW == 1 ? (D == 64 ? 4 : 3) : 2) void cache_attn_kernel(CacheAttnParams p) {
    constexpr int KC = D / 32, DT = D / 16, NP = sizeof(T) == 2 ? 1 : 3;
    constexpr int ROWB = D * 2, WAVE = (32 * ROWB > 16 * R * D * 4 ? 32 * ROWB : 16 * R * D * 4);    // values of a step; at the end a wave's sums
    __shared__ __attribute__((aligned(16))) uint8_t lds[4][WAVE];
    __shared__ float ends[4][2][16 * R];
    __shared__ uint32_t firsts[4][D];
    const int lane = threadIdx.x & 63, wave = threadIdx.x / 64, col = lane & 15, quarter = lane / 16;
    // Workgroups go to the eight dies in turn, so that neighbours are different heads and sequences, and all have as many: with a sequence's
    // chunks as neighbours the dies of the last ones idle where most sequences are short.
    const int units = p.c.count * p.c.KV * p.row_tiles, unit = blockIdx.x % units, chunk = blockIdx.x / units;
    const int b = unit / (p.c.KV * p.row_tiles), kv = unit / p.row_tiles % p.c.KV, row0 = unit % p.row_tiles * (16 * R), rows = p.fresh * p.group;
    const int seen = row_seen(p, b, min(row0 + 16 * R, rows) - 1), c0 = chunk * p.chunk;
    if (c0 >= seen && chunk > 0) return;
    const int c1 = min(c0 + p.chunk, seen);
    const bool alone = seen <= p.chunk;                  // the only chunk that there is

    // this lane's rows, and how far they see (rows that are not there: as far as any)
    int lim[R];
    i32x4_c q[R][NP][KC];
    float c = p.scale * 1.44269504f;
    const float flip = c < 0.0f ? -1.0f : c == 0.0f ? 0.0f : 1.0f;
    c = c < 0.0f ? -c : c == 0.0f ? 1.0f : c;
#pragma unroll
    for (int t = 0; t < R; ++t) {
        const int r = row0 + 16 * t + col, i = r / p.group, h = kv * p.group + r % p.group;
        const int64_t token = (int64_t)b * p.fresh + i;
        lim[t] = r < rows ? row_seen(p, b, r) : seen;
        const T* x = (const T*)p.Q + token * p.q.row + (int64_t)h * p.q.head + quarter * (D / 4);
#pragma unroll
        for (int k = 0; k < KC; ++k) {
            float v[8] = {0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f};
            if (r < rows) load_vec<8>(x + 8 * k, v);
            bf16_t piece[8][NP];
#pragma unroll
            for (int j = 0; j < 8; ++j) split<false>(flip == 0.0f ? 0.0f : v[j] * flip, piece[j]);
#pragma unroll
            for (int n = 0; n < NP; ++n)
#pragma unroll
                for (int j = 0; j < 4; ++j) q[t][n][k][j] = __builtin_bit_cast(int32_t, bf16x2_c{piece[2 * j][n], piece[2 * j + 1][n]});
        }
    }

    f32x4_c acc[R][DT];
    float top[R], sum[R];
#pragma unroll
    for (int t = 0; t < R; ++t) {
        top[t] = -__builtin_inff();
        sum[t] = 0.0f;
#pragma unroll
        for (int d = 0; d < DT; ++d) acc[t][d] = f32x4_c{0.0f, 0.0f, 0.0f, 0.0f};
    }
    int k0 = c0 + wave * 32;
    // Codes are loaded as soon as those of the step before are in use, the pages they are in a step ahead of that.  (Codes two steps ahead, with
    // two waves a SIMD fewer: no faster.)
    Part<D> nk[2], nv[2];
    bool there[2];
    int32_t page[2], column[2], line[2];                 // of the next step's positions: their page, its place in the table, their line in it
    const int columns = p.c.by_page.of(128), lines = 128 - columns * p.c.page;       // from one step to the next
    const uint64_t page_bytes = (uint64_t)p.c.KV * p.c.page * (D / 2), head_bytes = (uint64_t)kv * p.c.page * (D / 2);
    const int32_t* const pages = p.c.table + (int64_t)b * p.c.table_row;
    auto fetch = [&](int at0) {                          // codes of the step at at0, whose pages are known; then the next step's pages
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const int pos = at0 + 16 * u + col;
            there[u] = pos < c1 && (uint32_t)page[u] < (uint32_t)p.c.pages;
            const uint64_t at = page[u] * page_bytes + (head_bytes + __umul24(line[u], D / 2));
            nk[u].load(p.c.k, p.c.k_scale, there[u], at, quarter);
            nv[u].load(p.c.v, p.c.v_scale, there[u], at, quarter);
            column[u] += columns;
            line[u] += lines;
            if (line[u] >= p.c.page) { line[u] -= p.c.page; ++column[u]; }
            if (pos + 128 < c1) page[u] = pages[column[u]];
        }
    };
#pragma unroll
    for (int u = 0; u < 2; ++u) {
        const int pos = k0 + 16 * u + col;
        column[u] = p.c.by_page.of(pos);
        line[u] = pos - column[u] * p.c.page;
        page[u] = pos < c1 ? pages[column[u]] : -1;
    }
    fetch(k0);
    uint8_t* const mine = lds[wave];
    for (; k0 < c1; k0 += 128) {
        const uint32_t held = (uint32_t)(__ballot(there[0]) & 0xFFFF) | (uint32_t)((__ballot(there[1]) & 0xFFFF) << 16);       // positions that hold something
        const bool broken = (p.fresh > 1 || NW > 1) && __any(nv[0].broken() || nv[1].broken());
        // values to this wave's rows, after the reads of the step before
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (int u = 0; u < 2; ++u) {
#pragma unroll
            for (int k = 0; k < KC; ++k) {
                const int r = 16 * u + col;
                *(i32x4_c*)(mine + r * ROWB + ((quarter * KC + k) ^ value_turn<D>(r)) * 16) = nv[u].values(k);
            }
            __builtin_amdgcn_sched_barrier(0);           // (here and below: all of a step's conversions at once would cost a third of the waves)
        }
        __builtin_amdgcn_wave_barrier();
        f32x4_c s[R][2];
#pragma unroll
        for (int u = 0; u < 2; ++u) {
#pragma unroll
            for (int t = 0; t < R; ++t) s[t][u] = f32x4_c{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int k = 0; k < KC; ++k) {
                const i32x4_c a = nk[u].values(k);
#pragma unroll
                for (int t = 0; t < R; ++t)
#pragma unroll
                    for (int n = 0; n < NP; ++n) s[t][u] = product16(a, q[t][n][k], s[t][u]);
            }
            __builtin_amdgcn_sched_barrier(0);
        }
        fetch(k0 + 128);
        __builtin_amdgcn_sched_barrier(0);
        bool partly = held != 0xFFFFFFFFu;
        bool hidden = false;                             // a position that one row sees and another does not
#pragma unroll
        for (int t = 0; t < R; ++t) hidden |= lim[t] < min(k0 + 32, c1);
        hidden = __any(hidden);
        partly |= hidden;
        if (partly) {
#pragma unroll
            for (int t = 0; t < R; ++t)
#pragma unroll
                for (int u = 0; u < 2; ++u)
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        const int j = 16 * u + 4 * quarter + r;
                        if (k0 + j >= lim[t] || !((held >> j) & 1)) s[t][u][r] = -__builtin_inff();
                    }
        }
        bool move = false;
        float now[R];
#pragma unroll
        for (int t = 0; t < R; ++t) {
            float m = fmaxf(fmaxf(fmaxf(s[t][0][0], s[t][0][1]), fmaxf(s[t][0][2], s[t][0][3])), fmaxf(fmaxf(s[t][1][0], s[t][1][1]), fmaxf(s[t][1][2], s[t][1][3])));
            m = max_of_quarters(m) * c;
            now[t] = fmaxf(m, top[t]);
            move |= m > top[t] + 8.0f;
        }
        if (__any(move)) {
#pragma unroll
            for (int t = 0; t < R; ++t) {
                const float f = now[t] == -__builtin_inff() ? 1.0f : __builtin_amdgcn_exp2f(top[t] - now[t]);
                top[t] = now[t];
                sum[t] *= f;
#pragma unroll
                for (int d = 0; d < DT; ++d) acc[t][d] *= f;
            }
        }
        i32x4_c w[R][NW];
#pragma unroll
        for (int t = 0; t < R; ++t) {
            const float base = top[t] == -__builtin_inff() ? 0.0f : -top[t];
            bf16_t piece[8][NW];
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    s[t][u][r] = __builtin_amdgcn_exp2f(fmaf(s[t][u][r], c, base));
                    sum[t] += s[t][u][r];
                    split<true>(s[t][u][r], piece[4 * u + r]);
                }
#pragma unroll
            for (int n = 0; n < NW; ++n)
#pragma unroll
                for (int j = 0; j < 4; ++j) w[t][n][j] = __builtin_bit_cast(int32_t, bf16x2_c{piece[2 * j][n], piece[2 * j + 1][n]});
        }
        // infinities and NaN that some row does not see, or weights in pieces, the smaller of which are zero or negative
        const bool clean = broken && (hidden || NW > 1);
        if (clean) clean_values<D>(mine, firsts[wave]);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int d = 0; d < DT; ++d) {
            typedef __attribute__((address_space(3))) i16x4_c* lds_ptr;
            union { i16x4_c h[2]; i32x4_c v; } x;
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                const int r = 16 * u + 4 * quarter + col / 4;
                x.h[u] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr)(mine + r * ROWB + ((2 * d + (col & 3) / 2) ^ value_turn<D>(r)) * 16 + (col & 1) * 8));
            }
#pragma unroll
            for (int t = 0; t < R; ++t)
#pragma unroll
                for (int n = 0; n < NW; ++n) acc[t][d] = product16(x.v, w[t][n], acc[t][d]);
        }
        if (clean) {
#pragma unroll
            for (int t = 0; t < R; ++t) {
                const uint32_t rows = min(max(lim[t] - k0, 0), 32);
#pragma unroll
                for (int d = 0; d < DT; ++d) {
#pragma unroll
                    for (int r = 0; r < 4; ++r) acc[t][d][r] += broken_sum(firsts[wave][16 * d + 4 * quarter + r], rows);
                    __builtin_amdgcn_sched_barrier(0);   // (one after another: this is rare, and its registers would be everybody's)
                }
            }
        }
    }

    // the four waves' maxima, then their sums in one scale
#pragma unroll
    for (int t = 0; t < R; ++t) {
        sum[t] = sum_of_quarters(sum[t]);
        if (quarter == 0) { ends[wave][0][16 * t + col] = top[t]; ends[wave][1][16 * t + col] = sum[t]; }
    }
    __syncthreads();
    float* const sums = (float*)mine;
#pragma unroll
    for (int t = 0; t < R; ++t) {
        float m = ends[0][0][16 * t + col];
#pragma unroll
        for (int x = 1; x < 4; ++x) m = fmaxf(m, ends[x][0][16 * t + col]);
        const float f = m == -__builtin_inff() ? 0.0f : __builtin_amdgcn_exp2f(top[t] - m);
#pragma unroll
        for (int d = 0; d < DT; ++d) *(f32x4_c*)&sums[(16 * t + col) * D + ((4 * d + quarter) ^ (col & 7)) * 4] = acc[t][d] * f;
    }
    __syncthreads();
    for (int i = threadIdx.x; i < 16 * R * (D / 4); i += 256) {
        const int r = i / (D / 4), piece = i % (D / 4), row = row0 + r;
        if (row >= rows) continue;
        float m = ends[0][0][r];
#pragma unroll
        for (int x = 1; x < 4; ++x) m = fmaxf(m, ends[x][0][r]);
        f32x4_c v = {0.0f, 0.0f, 0.0f, 0.0f};
        float l = 0.0f;
#pragma unroll
        for (int x = 0; x < 4; ++x) {
            v += *(const f32x4_c*)&((const float*)lds[x])[r * D + (piece ^ (r & 7)) * 4];
            if (m != -__builtin_inff()) l = fmaf(ends[x][1][r], __builtin_amdgcn_exp2f(ends[x][0][r] - m), l);
        }
        const int64_t out = ((int64_t)b * p.fresh + row / p.group) * p.H + kv * p.group + row % p.group;
        if (alone) {
            const float inv = l == 0.0f ? 0.0f : 1.0f / l;
            const float o[4] = {v[0] * inv, v[1] * inv, v[2] * inv, v[3] * inv};
            if (p.o_type == LBA_F32) store_vec<4>((float*)p.O + out * D + piece * 4, o, p.fmt);
            else if (p.o_type == LBA_BF16) store_vec<4>((bf16_t*)p.O + out * D + piece * 4, o, p.fmt);
            else store_vec<4>((uint8_t*)p.O + out * D + piece * 4, o, p.fmt);
        } else {
            const int64_t to = out * p.chunks + chunk;
            *(f32x4_c*)&p.part[to * D + piece * 4] = v;
            if (piece == 0) {
                float* e = p.part + (int64_t)p.c.count * p.fresh * p.H * p.chunks * D + to * 2;
                e[0] = m;
                e[1] = l;
            }
        }
    }
}

template <typename T> void launch_cache_attn(const CacheAttnParams& p, int r, hipStream_t st) {
    const bool fine = sizeof(T) == 4 || p.fine;
    const dim3 grid((unsigned)p.chunks * (unsigned)(p.c.count * p.c.KV * p.row_tiles));
#define LBA_CACHE_ATTN(D_, R_) \
    if (p.c.D == D_ && r == R_) { \
        if (fine) hipLaunchKernelGGL((cache_attn_kernel<T, D_, R_, 3>), grid, dim3(256), 0, st, p); \
        else hipLaunchKernelGGL((cache_attn_kernel<T, D_, R_, sizeof(T) == 2 ? 1 : 3>), grid, dim3(256), 0, st, p); \
        return; \
    }
    LBA_CACHE_ATTN(32, 1) LBA_CACHE_ATTN(64, 1) LBA_CACHE_ATTN(96, 1) LBA_CACHE_ATTN(128, 1)
    LBA_CACHE_ATTN(32, 2) LBA_CACHE_ATTN(64, 2) LBA_CACHE_ATTN(96, 2) LBA_CACHE_ATTN(128, 2)
#undef LBA_CACHE_ATTN
}

}  // namespace lba
#endif

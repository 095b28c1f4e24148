// lba_attn_tile.h -- the tiles of the attention kernels: rows of heads in LDS, fragments of the matrix cores, which tile a workgroup has.
//
// A wave owns 32 columns of a product, one a lane pair (l, l + 32): the queries of S^T = K . Q^T and O^T = V^T . P^T, the keys of the backward
// pass's S = Q . K^T, dV^T = G^T . P and dK^T = Q^T . S.  The 32 x 32 result of a product has in lane l column l % 32 and in register r row
//   (r % 4) + 8 (r / 4) + 4 (l / 32),
// and the 16 x 32 factor of the next product needs of its 16 rows eight in each half of the wave: any eight, if the other factor is read in
// the same order.  So a result's registers 8 k .. 8 k + 7 are, rounded, the next factor's fragment as they are, what is per column (a query's
// maximum and sum) is per lane, and the other factor is read with rows (j % 4) + 8 (j / 4) + 4 (l / 32) of each 16: transposed reads of 4 x 16
// elements from LDS.
#ifndef LBA_ATTN_TILE_H_
#define LBA_ATTN_TILE_H_

#include <type_traits>

#include "lba_attn.h"

namespace lba {

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef float f32x4_t __attribute__((ext_vector_type(4)));
typedef int32_t i32x4_t __attribute__((ext_vector_type(4)));
typedef int16_t i16x4_t __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8_v __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2_v __attribute__((ext_vector_type(2)));

__device__ __attribute__((aligned(16))) const uint32_t attn_zeros[4] = {0, 0, 0, 0};

// eight elements of a factor's row
template <typename T> struct Frag;
template <> struct Frag<bf16_t> { i32x4_t w; };
template <> struct Frag<float> { f32x4_t a, b; };

// c + a . b of 32 x 16 and 16 x 32.  Float32: eight products of depth 2, the two halves of the wave one row each
__device__ __forceinline__ f32x16 product(const Frag<bf16_t>& a, const Frag<bf16_t>& b, f32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_v, a.w), __builtin_bit_cast(bf16x8_v, b.w), c, 0, 0, 0);
}
__device__ __forceinline__ f32x16 product(const Frag<float>& a, const Frag<float>& b, f32x16 c) {
#pragma unroll
    for (int j = 0; j < 4; ++j) c = __builtin_amdgcn_mfma_f32_32x32x2f32(a.a[j], b.a[j], c, 0, 0, 0);
#pragma unroll
    for (int j = 0; j < 4; ++j) c = __builtin_amdgcn_mfma_f32_32x32x2f32(a.b[j], b.b[j], c, 0, 0, 0);
    return c;
}

// the sum of the fragments' eight products
__device__ __forceinline__ float dot(const Frag<bf16_t>& a, const Frag<bf16_t>& b) {
    float s = 0.0f;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const uint32_t x = (uint32_t)a.w[j], y = (uint32_t)b.w[j];
        s = fmaf(__uint_as_float(x << 16), __uint_as_float(y << 16), s);
        s = fmaf(__uint_as_float(x & 0xFFFF0000u), __uint_as_float(y & 0xFFFF0000u), s);
    }
    return s;
}
__device__ __forceinline__ float dot(const Frag<float>& a, const Frag<float>& b) {
    float s = 0.0f;
#pragma unroll
    for (int j = 0; j < 4; ++j) s = fmaf(a.b[j], b.b[j], fmaf(a.a[j], b.a[j], s));
    return s;
}

// registers 8 k .. 8 k + 7 of a result as a fragment
template <typename T> __device__ __forceinline__ Frag<T> as_frag(const f32x16& s, int k) {
    Frag<T> f;
    if constexpr (sizeof(T) == 2) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const bf16x2_v two = {(bf16_t)s[8 * k + 2 * j], (bf16_t)s[8 * k + 2 * j + 1]};
            f.w[j] = __builtin_bit_cast(int32_t, two);
        }
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j) { f.a[j] = s[8 * k + j]; f.b[j] = s[8 * k + 4 + j]; }
    }
    return f;
}

// row of the result's register r in this lane's half
__device__ __forceinline__ constexpr int row_of(int r) { return (r % 4) + 8 * (r / 4); }

// ---- tiles in LDS ---------------------------------------------------------------------------
//
// A row of DP elements (D rounded up to 32, zeros behind D) is C = DP * sizeof(T) / 16 pieces of 16 bytes; piece c of row r stands at place
// c ^ turn(r) of its row.  Then the 16 lanes of a row read (one piece of 16 rows) and those of a transposed read (four pieces of four rows)
// meet 64 different banks.
template <int C> __device__ __forceinline__ int turn(int r) {
    if constexpr (C % 16 == 0) return ((r & 3) << 2) | ((r >> 2) & 3);
    else if constexpr (C % 8 == 0) return ((r & 2) << 1) | ((r >> 2) & 3);
    else return (r >> 2) & 3;
}

// the fragment of row `row` (this lane's) with elements 16 k + 8 (l / 32) ..
template <typename T, int DP> __device__ __forceinline__ Frag<T> row_frag(const uint8_t* tile, int row, int k, int half) {
    constexpr int C = DP * sizeof(T) / 16;
    const uint8_t* at = tile + row * (C * 16);
    Frag<T> f;
    if constexpr (sizeof(T) == 2) {
        f.w = *(const i32x4_t*)(at + ((2 * k + half) ^ turn<C>(row)) * 16);
    } else {
        f.a = *(const f32x4_t*)(at + ((4 * k + 2 * half) ^ turn<C>(row)) * 16);
        f.b = *(const f32x4_t*)(at + ((4 * k + 2 * half + 1) ^ turn<C>(row)) * 16);
    }
    return f;
}
// The fragment of column 32 t + l % 32 with rows row0 + (j % 4) + 8 (j / 4) + 4 (l / 32), row0 a multiple of 16.  A transposed read gives each of 16 lanes
// column i of a 4 x 16 block whose rows four lanes each address.
template <typename T, int DP> __device__ __forceinline__ Frag<T> column_frag(const uint8_t* tile, int row0, int t, int lane) {
    constexpr int C = DP * sizeof(T) / 16;
    Frag<T> f;
    if constexpr (sizeof(T) == 2) {
        const int r = row0 + 4 * (lane / 32) + (lane & 15) / 4, c = 4 * t + 2 * ((lane / 16) & 1) + (lane & 3) / 2;
        typedef __attribute__((address_space(3))) i16x4_t* lds_ptr;
        union { i16x4_t s[2]; i32x4_t w; } u;
#pragma unroll
        for (int i = 0; i < 2; ++i)
            u.s[i] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr)(tile + (r + 8 * i) * (C * 16) + (c ^ turn<C>(r + 8 * i)) * 16 + (lane & 1) * 8));
        f.w = u.w;
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int r = row0 + row_of(j) + 4 * (lane / 32);
            const float x = *(const float*)(tile + r * (C * 16) + ((8 * t + (lane & 31) / 4) ^ turn<C>(r)) * 16 + (lane & 3) * 4);
            if (j < 4) f.a[j] = x; else f.b[j - 4] = x;
        }
    }
    return f;
}
// 16 bytes a lane from memory to LDS, the wave's 64 pieces from the place `to` on.  Not the builtin: behind it the compiler waits for all that is under
// way before it reads LDS through a pointer that it cannot tell from the one written, the other buffer too (13 prompts forward 133 us with it,
// 128 so).  No register is written, nothing else here uses m0, and who reads the tile waits for vmcnt(0) and a barrier.
__device__ __forceinline__ void piece_to_lds(uint32_t to, const void* base, uint32_t offset) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(to), "v"(offset), "s"(base) : "memory");
}
__device__ __forceinline__ void piece_to_lds(uint32_t to, const void* from) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" ::"s"(to), "v"(from) : "memory");
}

// Rows of a head on their way to a tile of ROWS rows.  DIRECT: rows are whole pieces of 16 aligned bytes, a tile's rows within 2^31 bytes, and go
// from memory to LDS without registers in between; else a lane holds them until they are put down.  What is behind `rows` rows or D elements
// is zeros.
template <typename T, int DP, int ROWS, bool DIRECT> struct Loader {
    static constexpr int C = DP * sizeof(T) / 16, V = 16 / sizeof(T), N = ROWS * C / 256;
    static_assert(ROWS * C % 256 == 0, "whole pieces a lane");
    // 256 pieces are whole groups of 16 rows, after which turn() is the same: a lane's pieces are the same ones of rows 256 / C apart
    static constexpr bool EVEN = 4096 % (C * 256) == 0 && C <= 16;
    static constexpr int P = EVEN ? 1 : N;
    typedef typename Bits<T>::type B;
    const B* base;           // the next tile
    int64_t stride;
    typename std::conditional<DIRECT, uint32_t, int64_t>::type at[P];                // this lane's pieces in a tile: bytes, or elements, from its start
    int left[P];             // how many elements of the row are from there on
    bool full;               // rows have no pieces of zeros
    Raw<B, V> held[DIRECT ? 1 : N];

    __device__ __forceinline__ void start(const void* rows, int64_t row_stride, int D) {
        base = (const B*)rows;
        stride = row_stride;
        full = D == DP;
#pragma unroll
        for (int i = 0; i < P; ++i) {
            const int p = threadIdx.x + 256 * i, r = p / C, c = (p % C) ^ turn<C>(r);
            left[i] = D - c * V;
            at[i] = (r * row_stride + c * V) * (DIRECT ? (int)sizeof(T) : 1);
        }
    }
    // the next tile, of which `rows` rows are there
    __device__ __forceinline__ void load(uint8_t* tile, int rows) {
        if constexpr (DIRECT) {
            const uint32_t to = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint8_t*)tile + __builtin_amdgcn_readfirstlane(threadIdx.x / 64) * 1024;
            if (full && rows >= ROWS) {
#pragma unroll
                for (int i = 0; i < N; ++i) piece_to_lds(to + 4096 * i, EVEN ? base + i * (256 / C) * stride : base, at[EVEN ? 0 : i]);
            } else {
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    const bool in = ((int)threadIdx.x + 256 * i) / C < rows && left[EVEN ? 0 : i] > 0;
                    const char* src = (const char*)(EVEN ? base + i * (256 / C) * stride : base) + at[EVEN ? 0 : i];
                    piece_to_lds(to + 4096 * i, in ? (const void*)src : (const void*)attn_zeros);
                }
            }
        } else {
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const bool in = ((int)threadIdx.x + 256 * i) / C < rows;
                held[i] = load_raw<B, V>((EVEN ? base + i * (256 / C) * stride : base) + at[EVEN ? 0 : i], in ? left[EVEN ? 0 : i] : 0);
            }
        }
        base += stride * ROWS;
    }
    __device__ __forceinline__ void put(uint8_t* tile) const {
        if constexpr (!DIRECT) {
#pragma unroll
            for (int i = 0; i < N; ++i) *(i32x4_t*)(tile + (threadIdx.x + 256 * i) * 16) = __builtin_bit_cast(i32x4_t, held[i].v);
        }
    }
};

// Whether the tile holds an infinity or a NaN, looked for by the whole workgroup (a barrier: all of it calls).
template <typename T, int DP, int ROWS> __device__ __forceinline__ bool tile_is_broken(const uint8_t* tile) {
    constexpr int N = ROWS * DP * (int)sizeof(T) / 16 / 256;
    bool bad = false;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const i32x4_t w = *(const i32x4_t*)(tile + (threadIdx.x + 256 * i) * 16);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const uint32_t x = (uint32_t)w[j];
            if constexpr (sizeof(T) == 2) bad |= (x & 0x7F80u) == 0x7F80u || (x & 0x7F800000u) == 0x7F800000u;
            else bad |= (x & 0x7F800000u) == 0x7F800000u;
        }
    }
    return __syncthreads_or(bad) != 0;
}

// ---- tiles that hold infinities or NaN -----------------------------------------------------
//
// A product over rows some of which a column does not see must not multiply their infinities with its zeros.  Where a tile that is seen in part
// holds any, the weights' own NaN is enough for what is seen (dQ), or the workgroup's rows are done again, one by one over what each sees.

// the fragment with zeros for infinities and NaN
__device__ __forceinline__ Frag<bf16_t> without_broken(Frag<bf16_t> f) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const uint32_t x = (uint32_t)f.w[j];
        f.w[j] &= (int32_t)~(((x & 0x7F80u) == 0x7F80u ? 0xFFFFu : 0u) | ((x & 0x7F800000u) == 0x7F800000u ? 0xFFFF0000u : 0u));
    }
    return f;
}
__device__ __forceinline__ Frag<float> without_broken(Frag<float> f) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        f.a[j] = (__float_as_uint(f.a[j]) & 0x7F800000u) == 0x7F800000u ? 0.0f : f.a[j];
        f.b[j] = (__float_as_uint(f.b[j]) & 0x7F800000u) == 0x7F800000u ? 0.0f : f.b[j];
    }
    return f;
}
__device__ __forceinline__ float wave_max(float v) {
#pragma unroll
    for (int x = 32; x; x /= 2) v = fmaxf(v, __shfl_xor(v, x));
    return v;
}
// before a wave's own words of LDS are used for something else
__device__ __forceinline__ void wave_words_done() {
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_wave_barrier();
}

// a lane's row of a head as fragments: `D` elements from `at`, zeros behind; zeros where it is not there
template <typename T, int DP> __device__ __forceinline__ void load_frags(const void* at, bool there, int D, int half, Frag<T> (&f)[DP / 16]) {
    typedef typename Bits<T>::type B;
    const B* p = (const B*)at;
#pragma unroll
    for (int k = 0; k < DP / 16; ++k) {
        const int d = 16 * k + 8 * half;
        if constexpr (sizeof(T) == 2) {
            const Raw<B, 8> r = load_raw<B, 8>(p + d, there ? D - d : 0);
            f[k].w = __builtin_bit_cast(i32x4_t, r.v);
        } else {
            f[k].a = __builtin_bit_cast(f32x4_t, load_raw<B, 4>(p + d, there ? D - d : 0).v);
            f[k].b = __builtin_bit_cast(f32x4_t, load_raw<B, 4>(p + d + 4, there ? D - d - 4 : 0).v);
        }
    }
}

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

// the larger of a value's copies in lanes l and l ^ 32, and their sum: of the exchange's two results one is the wave's lower half twice, the other its
// upper half
__device__ __forceinline__ float max_of_halves(float v) {
    const auto x = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return fmaxf(__uint_as_float(x[0]), __uint_as_float(x[1]));
}
__device__ __forceinline__ float sum_of_halves(float v) {
    const auto x = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __uint_as_float(x[0]) + __uint_as_float(x[1]);
}

// store(pointer to O's type): O as what it is
template <typename F> __device__ __forceinline__ void with_output(const AttnParams& p, F store) {
    if (p.o_type == LBA_F32) store((float*)p.O);
    else if (p.o_type == LBA_BF16) store((bf16_t*)p.O);
    else store((uint8_t*)p.O);
}

// ---- rows of no sequence ----------------------------------------------------------------------

// the rows of no sequence, by the last blocks of the grid
template <typename T> __device__ __forceinline__ void clear_rows(const int32_t* starts, int T_rows, int count, int block, int blocks, T* out, int64_t row_stride,
                                                                 int64_t head_stride, int H, int D, float* lse, const CodeFmt& fmt) {
    const int first = count > 0 ? min(max(starts[0], 0), T_rows) : T_rows, last = count > 0 ? min(max(starts[count], first), T_rows) : T_rows;
    const int64_t rows = (int64_t)first + (T_rows - last);
    for (int64_t i = (int64_t)block * 256 + threadIdx.x; i < rows * H * D; i += (int64_t)blocks * 256) {
        const int d = (int)(i % D), h = (int)(i / D % H);
        const int64_t r = i / D / H, t = r < first ? r : last + (r - first);
        store_one(out + t * row_stride + h * head_stride + d, 0.0f, fmt);
        if (lse && d == 0) lse[t * H + h] = -__builtin_inff();
    }
}

// ---- which tile -----------------------------------------------------------------------------

struct TileOf {
    int b, t;                // sequence (-1: none) and its tile
    Rows mine, other;        // the sequence's rows in the list that has the tiles, and in the other one
};

// Tile `index` of the tiles of `size` rows that the sequences have one after another in `starts` (T rows); the whole wave calls.  Both lists are read
// at once, 64 sequences at a time: a workgroup waits for memory once before it knows its rows.
__device__ __forceinline__ TileOf find_tile(const int32_t* starts, int T, const int32_t* others, int T_other, int count, int size, int index) {
    if (!starts) {
        const int n = T / count, m = T_other / count, per = (n + size - 1) / size;
        if (per == 0 || index / per >= count) return {-1, 0, {0, 0}, {0, 0}};
        const int b = index / per;
        return {b, index % per, {b * n, n}, {b * m, m}};
    }
    const int lane = threadIdx.x & 63;
    for (int b0 = 0; b0 < count; b0 += 64) {
        const int b = min(b0 + lane, count - 1);
        const Rows mine = rows_of(starts, T, count, b), other = rows_of(others, T_other, count, b);
        const int n = b0 + lane < count ? (mine.n + size - 1) / size : 0;
        int upto = n;
#pragma unroll
        for (int x = 1; x < 64; x *= 2) {
            const int v = __shfl_up(upto, x);
            if (lane >= x) upto += v;
        }
        const uint64_t behind = __ballot(upto > index);
        if (behind) {
            const int f = __builtin_ctzll(behind);
            auto of = [&](int v) { return __builtin_amdgcn_readlane(v, f); };
            return {b0 + f, index - (of(upto) - of(n)), {of(mine.first), of(mine.n)}, {of(other.first), of(other.n)}};
        }
        index -= __builtin_amdgcn_readlane(upto, 63);
    }
    return {-1, 0, {0, 0}, {0, 0}};
}

// Part `slice` of what a workgroup does in n steps, cut into at most `slices` parts of two steps or more: steps first .. last - 1 (none in some of
// the later ones), `alone` where one part has them all.
struct Slice {
    int first, last;
    bool alone;
};
__device__ __forceinline__ int slice_steps(int n, int slices) { return max(2, (n + slices - 1) / slices); }
__device__ __forceinline__ Slice slice_of(int n, int slices, int slice) {
    const int per = slice_steps(n, slices);
    return {min(n, slice * per), min(n, slice * per + per), n <= per};
}
__device__ __forceinline__ int slices_used(int n, int slices) { return (n + slice_steps(n, slices) - 1) / slice_steps(n, slices); }

// how many keys query i of a sequence sees, and the first query that sees key j
__device__ __forceinline__ int keys_seen(const AttnParams& p, const Rows& rq, const Rows& rk, int i) { return p.causal ? max(0, min(rk.n, i + rk.n - rq.n + 1)) : rk.n; }
__device__ __forceinline__ int first_query(const AttnParams& p, const Rows& rq, const Rows& rk, int j) { return p.causal ? max(0, j - (rk.n - rq.n)) : 0; }
// steps of a tile of queries over tiles of `size` keys, and of a tile of keys over tiles of `size` queries of one head
__device__ __forceinline__ int steps_of_queries(const AttnParams& p, const Rows& rq, const Rows& rk, int t, int size) {
    return (keys_seen(p, rq, rk, min(t * kTileRows + kTileRows, rq.n) - 1) + size - 1) / size;
}
__device__ __forceinline__ int steps_of_keys(const AttnParams& p, const Rows& rq, const Rows& rk, int t, int size) {
    const int lo = first_query(p, rq, rk, t * kTileRows);
    return rq.n > lo ? (rq.n + size - 1) / size - lo / size : 0;
}
template <typename T> constexpr int kStep = sizeof(T) == 2 ? 64 : 32;                // keys or queries of a step

// how many tiles there may be
inline int64_t most_tiles(const int32_t* starts, int64_t T, int64_t count, int size) {
    if (count < 1 || T < 1) return 0;
    if (!starts) return count * ((T / count + size - 1) / size);
    return T / size + (count < T ? count : T);
}

// Workgroups go to the eight dies in turn; each die takes a run of neighbouring units, which share a head's keys in its cache.
__device__ __forceinline__ int unit_of(int block, int units) {
    const int per = units / 8, more = units % 8, die = block % 8;
    return die * per + min(die, more) + block / 8;
}

}  // namespace lba
#endif

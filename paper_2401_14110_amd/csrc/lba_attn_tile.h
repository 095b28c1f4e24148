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
typedef int32_t i32x2_t __attribute__((ext_vector_type(2)));
typedef int16_t i16x4_t __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8_v __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2_v __attribute__((ext_vector_type(2)));

__device__ __attribute__((aligned(16))) const uint32_t attn_zeros[4] = {0, 0, 0, 0};

// Eight elements of a factor's row.  Float32: in three bfloat16 pieces, which hold all 24 bits (of numbers of 2^-100 or more)
template <typename T> struct Frag;
template <> struct Frag<bf16_t> { i32x4_t w; };
template <> struct Frag<float> { i32x4_t w[3]; };

// Two numbers' pieces: the nearest bfloat16 number, that of what is left, and the rest.  Not FINITE: an infinity or a NaN is the last piece, with zeros before
// it, and first pieces stay within bfloat16, so that numbers that would round up to infinity do not get one.
template <bool FINITE> __device__ __forceinline__ void split_two(float x, float y, int32_t (&w)[3]) {
    constexpr float TOP = 3.38953139e38f;                // bfloat16's largest number
    const bool is[2] = {FINITE || fabsf(x) < __builtin_inff(), FINITE || fabsf(y) < __builtin_inff()};
    auto near = [&](float v, int i) { return FINITE ? v : is[i] ? __builtin_amdgcn_fmed3f(v, -TOP, TOP) : 0.0f; };
    const bf16x2_v a = {(bf16_t)near(x, 0), (bf16_t)near(y, 1)};
    x -= (float)a[0];
    y -= (float)a[1];
    const bf16x2_v b = {(bf16_t)near(x, 0), (bf16_t)near(y, 1)};
    const bf16x2_v c = {(bf16_t)(x - (float)b[0]), (bf16_t)(y - (float)b[1])};
    w[0] = __builtin_bit_cast(int32_t, a);
    w[1] = __builtin_bit_cast(int32_t, b);
    w[2] = __builtin_bit_cast(int32_t, c);
}
template <bool FINITE> __device__ __forceinline__ Frag<float> split_eight(const float (&x)[8]) {
    Frag<float> f;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        int32_t w[3];
        split_two<FINITE>(x[2 * j], x[2 * j + 1], w);
#pragma unroll
        for (int n = 0; n < 3; ++n) f.w[n][j] = w[n];
    }
    return f;
}

// c + a . b of 32 x 16 and 16 x 32.  Float32: the six products of pieces that are 2^-16 or more of the whole; the three others are under 2^-24 of it
// together.  (They take 192 cycles, float32's own instructions 512.)
__device__ __forceinline__ f32x16 product(const Frag<bf16_t>& a, const Frag<bf16_t>& b, f32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_v, a.w), __builtin_bit_cast(bf16x8_v, b.w), c, 0, 0, 0);
}
__device__ __forceinline__ f32x16 product(const Frag<float>& a, const Frag<float>& b, f32x16 c) {
#pragma unroll
    for (int n = 2; n >= 0; --n)
#pragma unroll
        for (int j = 0; j <= n; ++j) c = product(Frag<bf16_t>{a.w[j]}, Frag<bf16_t>{b.w[n - j]}, c);
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
    auto low = [](const Frag<float>& f, int j) { return (__uint_as_float((uint32_t)f.w[2][j] << 16) + __uint_as_float((uint32_t)f.w[1][j] << 16)) + __uint_as_float((uint32_t)f.w[0][j] << 16); };
    auto high = [](const Frag<float>& f, int j) {
        return (__uint_as_float((uint32_t)f.w[2][j] & 0xFFFF0000u) + __uint_as_float((uint32_t)f.w[1][j] & 0xFFFF0000u)) + __uint_as_float((uint32_t)f.w[0][j] & 0xFFFF0000u);
    };
    float s = 0.0f;
#pragma unroll
    for (int j = 0; j < 4; ++j) s = fmaf(high(a, j), high(b, j), fmaf(low(a, j), low(b, j), s));
    return s;
}

// registers 8 k .. 8 k + 7 of a result as a fragment
template <typename T> __device__ __forceinline__ Frag<T> as_frag(const f32x16& s, int k) {
    if constexpr (sizeof(T) == 2) {
        Frag<T> f;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const bf16x2_v two = {(bf16_t)s[8 * k + 2 * j], (bf16_t)s[8 * k + 2 * j + 1]};
            f.w[j] = __builtin_bit_cast(int32_t, two);
        }
        return f;
    } else {
        float x[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) x[j] = s[8 * k + j];
        return split_eight<true>(x);
    }
}

// The same as `N` bfloat16 factors: the numbers rounded, or (3) pieces that hold them.
template <int N> __device__ __forceinline__ void as_factors(const f32x16& s, int k, Frag<bf16_t> (&f)[N]) {
    if constexpr (N == 1) {
        f[0] = as_frag<bf16_t>(s, k);
    } else {
        const Frag<float> x = as_frag<float>(s, k);
#pragma unroll
        for (int n = 0; n < N; ++n) f[n].w = x.w[n];
    }
}

// row of the result's register r in this lane's half
__device__ __forceinline__ constexpr int row_of(int r) { return (r % 4) + 8 * (r / 4); }

// ---- tiles in LDS ---------------------------------------------------------------------------
//
// A row of DP elements (D rounded up to 32, zeros behind D) is C = DP / 8 pieces of 16 bytes; piece c of row r stands at place c ^ turn(r) of its row.
// Then the 16 lanes of a row read (one piece of 16 rows) and those of a transposed read (four pieces of four rows) meet 64 different banks.
// Float32: three such tiles one behind another, of the numbers' first, second and third pieces.
template <int C> __device__ __forceinline__ int turn(int r) {
    if constexpr (C % 16 == 0) return ((r & 3) << 2) | ((r >> 2) & 3);
    else if constexpr (C % 8 == 0) return ((r & 2) << 1) | ((r >> 2) & 3);
    else return (r >> 2) & 3;
}
template <typename T> constexpr int kStep = sizeof(T) == 2 ? 64 : 32;                // rows of a tile: keys or queries of a step
template <typename T> constexpr int kPieces = sizeof(T) == 2 ? 1 : 3;
template <typename T, int DP> constexpr int kTileBytes = kStep<T> * DP * 2 * kPieces<T>;

// the fragment of row `row` (this lane's) with elements 16 k + 8 (l / 32) ..
template <typename T, int DP> __device__ __forceinline__ Frag<T> row_frag(const uint8_t* tile, int row, int k, int half) {
    constexpr int C = DP / 8;
    const uint8_t* at = tile + row * (C * 16) + ((2 * k + half) ^ turn<C>(row)) * 16;
    Frag<T> f;
    if constexpr (sizeof(T) == 2) {
        f.w = *(const i32x4_t*)at;
    } else {
#pragma unroll
        for (int n = 0; n < 3; ++n) f.w[n] = *(const i32x4_t*)(at + n * (kTileBytes<T, DP> / 3));
    }
    return f;
}
// The fragment of column 32 t + l % 32 with rows row0 + (j % 4) + 8 (j / 4) + 4 (l / 32), row0 a multiple of 16.  A transposed read gives each of 16 lanes
// column i of a 4 x 16 block whose rows four lanes each address.
template <typename T, int DP> __device__ __forceinline__ Frag<T> column_frag(const uint8_t* tile, int row0, int t, int lane) {
    constexpr int C = DP / 8;
    const int r = row0 + 4 * (lane / 32) + (lane & 15) / 4, c = 4 * t + 2 * ((lane / 16) & 1) + (lane & 3) / 2;
    auto columns = [&](const uint8_t* at) {
        typedef __attribute__((address_space(3))) i16x4_t* lds_ptr;
        union { i16x4_t s[2]; i32x4_t w; } u;
#pragma unroll
        for (int i = 0; i < 2; ++i)
            u.s[i] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr)(at + (r + 8 * i) * (C * 16) + (c ^ turn<C>(r + 8 * i)) * 16 + (lane & 1) * 8));
        return u.w;
    };
    Frag<T> f;
    if constexpr (sizeof(T) == 2) {
        f.w = columns(tile);
    } else {
#pragma unroll
        for (int n = 0; n < 3; ++n) f.w[n] = columns(tile + n * (kTileBytes<T, DP> / 3));
    }
    return f;
}
// 16 bytes a lane from memory to LDS, the wave's 64 pieces from the place `to` on.  Not the builtin: behind it the compiler waits for all that is under
// way before it reads LDS through a pointer that it cannot tell from the one written, the other buffer too (13 prompts forward 133 us with it,
// 128 so).  No register is written but m0, which the compiler reserves (it takes no mention of it among what is changed): it sets m0 right before an
// instruction of its own that reads it, and these kernels have none.  Who reads the tile waits for vmcnt(0) and a barrier.
__device__ __forceinline__ void piece_to_lds(uint32_t to, const void* base, uint32_t offset) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(to), "v"(offset), "s"(base) : "memory");
}
__device__ __forceinline__ void piece_to_lds(uint32_t to, const void* from) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" ::"s"(to), "v"(from) : "memory");
}

// The end of a row that is no whole vector: the row's last V elements are loaded, and moved down by those that belong to the vector before, once
// they are there.  (One by one they would be waited for where they are loaded, and with them all that is under way.)
template <typename B, int V> __device__ __forceinline__ Raw<B, V> load_all(const B* p, bool there) {
    Raw<B, V> r = {};
    if (there) r.v = *(const typename Vec<B, V>::type*)p;
    return r;
}
// the first `n` of fewer than V elements (a loop: such heads are rare, and this stands wherever a tile is loaded)
template <typename B, int V> __device__ __forceinline__ Raw<B, V> load_few(const B* p, int n) {
    i32x4_t w = {0, 0, 0, 0};
#pragma clang loop unroll(disable)
    for (int j = n - 1; j >= 0; --j) {
        if constexpr (sizeof(B) == 2) {
            w = i32x4_t{w[0] << 16, (int32_t)__builtin_amdgcn_alignbit(w[1], w[0], 16), (int32_t)__builtin_amdgcn_alignbit(w[2], w[1], 16),
                        (int32_t)__builtin_amdgcn_alignbit(w[3], w[2], 16)};
            w[0] |= p[j];
        } else {
            w = i32x4_t{(int32_t)__float_as_uint(p[j]), w[0], w[1], w[2]};
        }
    }
    Raw<B, V> r;
    r.v = __builtin_bit_cast(decltype(r.v), w);
    return r;
}
template <typename B, int V> __device__ __forceinline__ int before_end(int left) { return left > 0 && left < V ? V - left : 0; }
template <typename B, int V> __device__ __forceinline__ void move_down(Raw<B, V>& r, int by) {
    i32x4_t w = __builtin_bit_cast(i32x4_t, r.v);
    int step = by;
    if constexpr (sizeof(B) == 2) {
        const i32x4_t m = {(int32_t)__builtin_amdgcn_alignbit(w[1], w[0], 16), (int32_t)__builtin_amdgcn_alignbit(w[2], w[1], 16),
                           (int32_t)__builtin_amdgcn_alignbit(w[3], w[2], 16), (int32_t)((uint32_t)w[3] >> 16)};
        w = step & 1 ? m : w;
        step >>= 1;
    }
    w = step & 1 ? i32x4_t{w[1], w[2], w[3], 0} : w;
    w = step & 2 ? i32x4_t{w[2], w[3], 0, 0} : w;
    r.v = __builtin_bit_cast(decltype(r.v), w);
}

// Rows of a head on their way to a tile.  DIRECT: rows are whole pieces of 16 aligned bytes of bfloat16, a tile's rows within 2^31 bytes, and go from
// memory to LDS without registers in between; else a lane holds 16 bytes each until they are put down.  What is behind `rows` rows or D
// elements is zeros.
template <typename T, int DP, bool DIRECT> struct Loader {
    static constexpr int ROWS = kStep<T>, C = DP * sizeof(T) / 16, V = 16 / sizeof(T), N = ROWS * C / 256;
    static_assert(ROWS * C % 256 == 0 && !(DIRECT && sizeof(T) != 2), "whole pieces a lane");
    // 256 pieces are whole groups of 16 rows, after which turn() is the same: a lane's pieces are the same ones of rows 256 / C apart
    static constexpr bool EVEN = 4096 % (C * 256) == 0 && C <= 16;
    static constexpr int P = EVEN ? 1 : N;
    typedef typename Bits<T>::type B;
    const B* base;           // the next tile
    int64_t stride;
    typename std::conditional<DIRECT, uint32_t, int64_t>::type at[P];                // this lane's pieces in a tile: bytes, or elements, from its start
    int left[P];             // how many elements of the row are from there on
    int down[P];             // not DIRECT: by how many elements a piece is moved down
    bool full;               // rows have no pieces of zeros
    bool ragged, tiny;       // not DIRECT: rows end inside a piece, the first one
    Raw<B, V> held[DIRECT ? 1 : N];

    __device__ __forceinline__ void start(const void* rows, int64_t row_stride, int D) {
        base = (const B*)rows;
        stride = row_stride;
        full = D == DP;
#pragma unroll
        for (int i = 0; i < P; ++i) {
            const int p = threadIdx.x + 256 * i, r = p / C, c = sizeof(T) == 2 ? (p % C) ^ turn<C>(r) : p % C;
            left[i] = D - c * V;
            down[i] = DIRECT || D < V ? 0 : before_end<B, V>(left[i]);
            at[i] = (r * row_stride + c * V - down[i]) * (DIRECT ? (int)sizeof(T) : 1);
        }
        ragged = D % V != 0 && D >= V;
        tiny = D < V;
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
                const B* src = (EVEN ? base + i * (256 / C) * stride : base) + at[EVEN ? 0 : i];
                if (tiny) held[i] = load_few<B, V>(src, in ? left[EVEN ? 0 : i] : 0);
                else held[i] = load_all<B, V>(src, in && left[EVEN ? 0 : i] > 0);
            }
        }
        base += stride * ROWS;
    }
    __device__ __forceinline__ void put(uint8_t* tile) {
        if constexpr (!DIRECT) {
            if (ragged) {
#pragma unroll
                for (int i = 0; i < N; ++i) move_down<B, V>(held[i], down[EVEN ? 0 : i]);
            }
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const int p = threadIdx.x + 256 * i;
                if constexpr (sizeof(T) == 2) {
                    *(i32x4_t*)(tile + p * 16) = __builtin_bit_cast(i32x4_t, held[i].v);
                } else {                                 // four numbers: half a piece of each tile
                    const f32x4_t x = __builtin_bit_cast(f32x4_t, held[i].v);
                    const int r = p / C, c = p % C;
                    uint8_t* const at = tile + r * (DP * 2) + ((c / 2) ^ turn<DP / 8>(r)) * 16 + (c & 1) * 8;
                    int32_t a[3], b[3];
                    split_two<false>(x[0], x[1], a);
                    split_two<false>(x[2], x[3], b);
#pragma unroll
                    for (int n = 0; n < 3; ++n) *(i32x2_t*)(at + n * (kTileBytes<T, DP> / 3)) = i32x2_t{a[n], b[n]};
                }
            }
        }
    }
};

// Whether the tile holds an infinity or a NaN (float32: its last pieces do), looked for by the whole workgroup (a barrier: all of it calls).
template <typename T, int DP> __device__ __forceinline__ bool tile_is_broken(const uint8_t* tile) {
    bool bad = false;
#pragma unroll
    for (int i = threadIdx.x; i < kStep<T> * DP / 8; i += 256) {
        const i32x4_t w = *(const i32x4_t*)(tile + (kPieces<T> - 1) * (kTileBytes<T, DP> / kPieces<T>) + i * 16);
#pragma unroll
        for (int j = 0; j < 4; ++j) bad |= ((uint32_t)w[j] & 0x7F80u) == 0x7F80u || ((uint32_t)w[j] & 0x7F800000u) == 0x7F800000u;
    }
    return __syncthreads_or(bad) != 0;
}

// ---- tiles that hold infinities or NaN -----------------------------------------------------
//
// A product over rows some of which a column does not see must not multiply their infinities with its zeros.  Where a tile that is seen in part
// holds any, zeros stand for them; what they do to columns that see them comes from elsewhere: the weights' own NaN (gradients), or where they are.

// the fragment with zeros for infinities and NaN
__device__ __forceinline__ Frag<bf16_t> without_broken(Frag<bf16_t> f) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const uint32_t x = (uint32_t)f.w[j];
        f.w[j] &= (int32_t)~(((x & 0x7F80u) == 0x7F80u ? 0xFFFFu : 0u) | ((x & 0x7F800000u) == 0x7F800000u ? 0xFFFF0000u : 0u));
    }
    return f;
}
__device__ __forceinline__ Frag<float> without_broken(Frag<float> f) {                // (the other pieces of such are zeros)
    f.w[2] = without_broken(Frag<bf16_t>{f.w[2]}).w;
    return f;
}
__device__ __forceinline__ float wave_max(float v) {
#pragma unroll
    for (int x = 32; x; x /= 2) v = fmaxf(v, __shfl_xor(v, x));
    return v;
}
// The same of a tile in LDS, by the whole workgroup: a barrier before, when all have read it, and after.
template <typename T, int DP> __device__ __forceinline__ void clean_tile(uint8_t* tile) {
    __syncthreads();
    for (int i = threadIdx.x; i < kStep<T> * DP / 8; i += 256) {
        i32x4_t* const at = (i32x4_t*)(tile + (kPieces<T> - 1) * (kTileBytes<T, DP> / kPieces<T>) + i * 16);
        *at = without_broken(Frag<bf16_t>{*at}).w;
    }
    __syncthreads();
}

// What infinities and NaN in a tile do to sums over its rows is known by a column's first row with each of them, since a query sees the first rows of a
// tile: firsts[d] has that of infinity, of its negative and of NaN in a byte each (64: there is none).  The whole workgroup calls, clean_tile comes next.
template <typename T, int DP> __device__ __forceinline__ void find_broken(const uint8_t* tile, uint32_t* firsts) {
    const uint8_t* const last = tile + (kPieces<T> - 1) * (kTileBytes<T, DP> / kPieces<T>);
    const int d = threadIdx.x;
    if (d >= DP) return;
    uint32_t plus = 64, minus = 64, none = 64;
#pragma clang loop unroll(disable)
    for (int row = kStep<T> - 1; row >= 0; --row) {
        const uint32_t e = *(const uint16_t*)(last + row * (DP * 2) + ((d / 8) ^ turn<DP / 8>(row)) * 16 + d % 8 * 2);
        if (e == 0x7F80u) plus = row;
        if (e == 0xFF80u) minus = row;
        if ((e & 0x7FFFu) > 0x7F80u) none = row;
    }
    firsts[d] = plus | minus << 8 | none << 16;
}
// what is added to a column of which `seen` rows are seen
__device__ __forceinline__ float broken_sum(uint32_t firsts, uint32_t seen) {
    const bool plus = (firsts & 255) < seen, minus = ((firsts >> 8) & 255) < seen, none = firsts >> 16 < seen;
    return none || (plus && minus) ? __builtin_nanf("") : plus ? __builtin_inff() : minus ? -__builtin_inff() : 0.0f;
}

// a lane's row of a head as fragments: `D` elements from `at`, zeros behind; zeros where it is not there
template <typename T, int DP> __device__ __forceinline__ void load_frags(const void* at, bool there, int D, int half, Frag<T> (&f)[DP / 16]) {
    typedef typename Bits<T>::type B;
    constexpr int V = 16 / sizeof(T), N = 8 / V;         // N vectors a fragment
    const B* p = (const B*)at;
    Raw<B, V> r[DP / 16][N];
#pragma unroll
    for (int k = 0; k < DP / 16; ++k)
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int d = 16 * k + 8 * half + V * i, left = there ? D - d : 0;
            if (D < V) r[k][i] = load_few<B, V>(p + d, left);
            else r[k][i] = load_all<B, V>(p + d - before_end<B, V>(left), left > 0);
        }
    if (D % V != 0 && D >= V) {
#pragma unroll
        for (int k = 0; k < DP / 16; ++k)
#pragma unroll
            for (int i = 0; i < N; ++i) move_down<B, V>(r[k][i], before_end<B, V>(D - 16 * k - 8 * half - V * i));
    }
#pragma unroll
    for (int k = 0; k < DP / 16; ++k) {
        if constexpr (sizeof(T) == 2) {
            f[k].w = __builtin_bit_cast(i32x4_t, r[k][0].v);
        } else {
            const f32x4_t a = __builtin_bit_cast(f32x4_t, r[k][0].v), b = __builtin_bit_cast(f32x4_t, r[k][1].v);
            const float x[8] = {a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]};
            f[k] = split_eight<false>(x);
        }
    }
}

// The fragments are there from here on.  Else the compiler waits for their loads where they are first used, in a loop at every turn, and there for all
// that is under way, the next tile too (dK and dV of 2 sequences of 4096, 32 heads of 128 on 8: 713 us so, 669 with this).
template <int N> __device__ __forceinline__ void arrived(Frag<bf16_t> (&f)[N]) {
#pragma unroll
    for (int k = 0; k < N; ++k) asm volatile("" : "+v"(f[k].w));
}
template <int N> __device__ __forceinline__ void arrived(Frag<float> (&f)[N]) {
#pragma unroll
    for (int k = 0; k < N; ++k) asm volatile("" : "+v"(f[k].w[0]), "+v"(f[k].w[1]), "+v"(f[k].w[2]));
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

// The last sequence of 0 .. count - 1 whose `key`, which never falls from one to the next, is not behind `at`, with its rows in both lists (b = -1: there is none);
// the whole wave calls.  64 keys at a time, then 64 sequences' rows at once: three reads one after another for 2^18 sequences.
template <typename K> __device__ __forceinline__ TileOf find_last(const int32_t* starts, int T, const int32_t* others, int T_other, int count, int at, K key) {
    const int lane = threadIdx.x & 63;
    int lo = 0, hi = count;                              // it is one of lo .. hi - 1, if any
    while (hi - lo > 64) {
        const int step = (hi - lo + 63) / 64, b = lo + lane * step;
        const uint64_t before = __ballot(b < hi && key(min(b, hi - 1)) <= at);
        if (before) lo += (63 - __builtin_clzll(before)) * step;
        hi = min(hi, lo + step);
    }
    const int b = min(lo + lane, hi - 1);
    const Rows mine = rows_of(starts, T, count, b), other = rows_of(others, T_other, count, b);
    const uint64_t before = __ballot(lo + lane < hi && key(b) <= at);
    if (!before) return {-1, 0, {0, 0}, {0, 0}};
    const int f = 63 - __builtin_clzll(before);
    auto of = [&](int v) { return __builtin_amdgcn_readlane(v, f); };
    return {of(b), 0, {of(mine.first), of(mine.n)}, {of(other.first), of(other.n)}};
}

constexpr int kPacked = 64;                              // sequences of a list up to which tiles have no gaps

// Tile `index` of the tiles of `size` rows that the sequences have in `starts` (T rows); the whole wave calls.  Up to kPacked sequences have theirs one
// after another, found by one look at both lists, a sequence a lane: a workgroup waits for memory once before it knows its rows.  Of more, sequence b has its from
// starts[b] / size + b on, where they fit whatever the others are, so that they can be searched for; the places between are nobody's.  (One after another, every
// workgroup walked over the list: 5000 sequences of one token, 4 heads, forward 780 us, 2^17 with one head 145 ms; so 141 us and 0.9 ms.)
__device__ __forceinline__ TileOf find_tile(const int32_t* starts, int T, const int32_t* others, int T_other, int count, int size, int index) {
    if (!starts) {
        const int n = T / count, m = T_other / count, per = (n + size - 1) / size;
        if (per == 0 || index / per >= count) return {-1, 0, {0, 0}, {0, 0}};
        const int b = index / per;
        return {b, index % per, {b * n, n}, {b * m, m}};
    }
    if (count > kPacked) {
        auto place = [&](int b) { return min(max(starts[b], 0), T) / size + b; };
        TileOf at = find_last(starts, T, others, T_other, count, index, place);
        if (at.b < 0) return at;
        at.t = index - (at.mine.first / size + at.b);
        if (at.t >= (at.mine.n + size - 1) / size) at.b = -1;
        return at;
    }
    const int lane = threadIdx.x & 63, b = min(lane, count - 1);
    const Rows mine = rows_of(starts, T, count, b), other = rows_of(others, T_other, count, b);
    const int n = lane < count ? (mine.n + size - 1) / size : 0;
    int upto = n;
#pragma unroll
    for (int x = 1; x < 64; x *= 2) {
        const int v = __shfl_up(upto, x);
        if (lane >= x) upto += v;
    }
    const uint64_t behind = __ballot(upto > index);
    if (!behind) return {-1, 0, {0, 0}, {0, 0}};
    const int f = __builtin_ctzll(behind);
    auto of = [&](int v) { return __builtin_amdgcn_readlane(v, f); };
    return {f, index - (of(upto) - of(n)), {of(mine.first), of(mine.n)}, {of(other.first), of(other.n)}};
}

// The sequence that row `t` of T belongs to in `starts`, with t as the tile; the whole wave calls.
__device__ __forceinline__ TileOf find_row(const int32_t* starts, int T, const int32_t* others, int T_other, int count, int t) {
    if (count < 1) return {-1, 0, {0, 0}, {0, 0}};
    if (!starts) {
        const int n = T / count, m = T_other / count, b = t / n;
        return {b, t, {b * n, n}, {b * m, m}};
    }
    TileOf at = find_last(starts, T, others, T_other, count, t, [&](int b) { return starts[b]; });
    if (at.b >= 0 && (t < at.mine.first || t >= at.mine.first + at.mine.n)) at.b = -1;
    at.t = t;
    return at;
}

// Elements `lane` and lane + 64 of `heads` (1 or 2) neighbouring heads of a row, of n parts `stride` apart times their weights: v = the sums.  All loads of
// four parts are on their way at once: what another workgroup has just stored is a microsecond away.
template <typename F> __device__ __forceinline__ void sum_parts(const float* part, int64_t stride, int n, int heads, int D, F weight, float (&v)[2][2]) {
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int h = 0; h < 2; ++h) v[h][0] = v[h][1] = 0.0f;
    for (int x0 = 0; x0 < n; x0 += 4) {
        float y[4][2][2];
#pragma unroll
        for (int x = 0; x < 4; ++x)
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int i = 0; i < 2; ++i) y[x][h][i] = part[min(x0 + x, n - 1) * stride + (h < heads ? h : 0) * D + min(lane + 64 * i, D - 1)];
#pragma unroll
        for (int x = 0; x < 4; ++x) {
            if (x0 + x >= n) break;
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int i = 0; i < 2; ++i) v[h][i] = fmaf(weight(h, x0 + x), y[x][h][i], v[h][i]);
        }
    }
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

// how many tiles there may be
inline int64_t most_tiles(const int32_t* starts, int64_t T, int64_t count, int size) {
    if (count < 1 || T < 1) return 0;
    if (!starts) return count * ((T / count + size - 1) / size);
    return T / size + (count < T || count > kPacked ? count : T);
}

// Workgroups go to the eight dies in turn; each die takes a run of neighbouring units, which share a head's keys (or queries) in its cache: 2 sequences of
// 4096, 32 heads of 128 on 8, forward 285 us, dQ 382, dK and dV 713, with units in turn 338, 457 and 1159.  (Cut into parts there are few workgroups,
// which then are in turn, so that all dies have as many.)
__device__ __forceinline__ int unit_of(int block, int units) {
    const int per = units / 8, more = units % 8, die = block % 8;
    return die * per + min(die, more) + block / 8;
}

}  // namespace lba
#endif

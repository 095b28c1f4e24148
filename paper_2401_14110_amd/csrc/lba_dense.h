// lba_dense.h -- the dense product's tile on the matrix cores, its epilogues and parameter blocks.
//
//   out[m, n] = sum_k A[m, k] * B[n, k]          both operands with k contiguous, 8-bit codes or bfloat16 elements
//
// The gfx950 matrix instructions on FP8 operands do not hold their sums in float32: within one instruction a product that is more than
// 13 binades below the largest one is dropped (measured with single products against one of 2^16; the same for the 16 x 16 x 32, 16 x 16 x 128
// and 32 x 32 x 64 forms).  On bfloat16 and FP16 operands the sum is float32's, subnormal operands included.  So codes travel as bytes through
// LDS and become bfloat16 (E4M3, one conversion instruction for two codes) or FP16 numbers (at most 4 exponent bits: the code's fields moved to
// FP16's places, which is the value times a power of two) in registers on their way into the matrix cores: products are exact, sums float32.
// A workgroup owns BM x BN outputs and walks over k in steps of 128 bytes of a row: BM + BN rows of the step go from global memory
// straight to LDS (16 bytes a lane, no registers in between) into one of NST buffers while the matrix cores work on another.
// A row of 128 bytes is 8 pieces of 16; piece c of row r stands at place c ^ (r / 2 % 8), so that the sixteen rows of a fragment
// read, 16 bytes each, fall on all 64 banks once.  An operand's pieces beyond the end of its rows are read from a zero page and
// rows beyond the last one repeat it: their outputs are not stored.
// Conversions and products do not overlap on a SIMD, whichever waves they belong to: a step takes their sum (256 x 256: 4096 cycles of
// products and 1800 of conversions take 5900), so the largest wave tile that its registers allow converts least.
// Fragments: lane l holds row l % 16 and pieces l / 16 and l / 16 + 4 of the step, the same places of k for both operands, so it does
// not matter in which order the matrix core walks over them.  B is the first factor, so lane l ends up with output row l % 16 and
// four neighbouring columns 4 * (l / 16) ..; the epilogue takes the sums through LDS, eight columns a lane.
// Measured: 8192 x 8192 x 4096 E4M3 with GELU to codes 397 to 417 us, 1.35 PFLOP/s (360 to 367 us, 1.5, without the activation; a library product of
// bfloat16 numbers reaches 1.34 to 1.37 at 8192^3); 4096 x 2304 x 768 to bfloat16 22 us, 0.65 (198 tiles on 256 CUs, six steps); 3136 x 512 x 4608 on
// M4E3 34 us, 0.43; 4096 x (2 x 4096) x 1024 gated 71 us, 0.97.  The gradients' products of bfloat16 rows are bound by LDS as much as by the
// matrix cores: 4096 x 8192 x 1024, both, 119 us and 11 to join the slices, 1.15; with float32 gradients, three pieces, 8192 x 2048 x 2048, both,
// 309 us, 1.33.
// Steps of half the length in four buffers instead of two took 9 to 30 % longer for bfloat16 rows.
#ifndef LBA_DENSE_H_
#define LBA_DENSE_H_

#include "lba_layer_device.h"
#include "lba_dense_index.h"

namespace lba {

typedef int32_t i32x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4_any __attribute__((ext_vector_type(4), aligned(2)));
typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8_t __attribute__((ext_vector_type(8)));

// what is done with the four neighbouring sums of a lane
struct EpiParams {
    float scale;             // of the raw sums
    const float* bias;       // [N], gated [2 N], or null
    int32_t act;
    DropParams drop;
    int32_t M, N;            // outputs (gated: of one half)
    // forward
    const void* R;
    int32_t r_type;
    void* Y;
    int32_t y_type;
    CodeFmt fmt;
    // backward: the gradient of the sums, as bfloat16 pieces in both orders, and its column sums
    const void* G;
    int32_t g_type;
    int32_t pieces;          // 1: rounded to bfloat16; 3: float32 split exactly
    bf16_t* P;               // [pieces][M][ldp]: N columns and zeros up to `wide`, gated: then the second half's
    bf16_t* PT;              // [pieces][N or 2 N][ldt]
    int64_t ldp, ldt, p_piece, pt_piece;
    int32_t wide;            // N rounded up to 8
    float* part;             // [rows of partial sums][N or 2 N], or null
};

struct GemmParams {
    const uint8_t* A;
    const uint8_t* B;
    int64_t lda, ldb;        // bytes from row to row
    int64_t a_piece;         // bytes from piece to piece of A where it comes in three
    int32_t rows_a, rows_b;
    int32_t half;            // gated: first row of B's second half
    int32_t chunks;          // 16-byte pieces of a row
    int32_t steps;           // steps of a row: of 128 bytes, of 64 where A comes in three pieces
    int32_t gx, gy;          // tiles over m and n
    int32_t slices;          // > 1: the steps are cut into so many slices of `per_slice`, each of which stores its sums in `split`
    int32_t per_slice;
    float* split;            // [slices][M][rows_b] raw sums
    int32_t shift_a, shift_b;     // ELEM_F16: M - 2 of the operand's format
    uint32_t keep_a, keep_b;      // and the places of sign and magnitude in both halves of a word
    EpiParams e;
};

// code -> value at the canonical bias 2^(E-1) - 1, exact (at most 6 significant bits: a bfloat16 number)
struct CodeBits { int32_t sh; uint32_t exp0, sub; float two; };   // 23 - M, (127 - bias) << 23, 1 << M, 2^(1 - bias)
inline CodeBits make_code_bits(const lba_infmt& f) {
    const int bc = (1 << (f.exp_bits - 1)) - 1;
    return {23 - f.man_bits, (uint32_t)(127 - bc) << 23, 1u << f.man_bits, __builtin_ldexpf(1.0f, 1 - bc)};
}
__device__ __forceinline__ float code_value(uint32_t code, const CodeBits& b) {
    const uint32_t mag = code & 0x7Fu;
    float f = __uint_as_float((mag << b.sh) + b.exp0);
    if (mag < b.sub) f = fmaf(2.0f, f, -b.two);          // subnormal: the leading one does not count
    return __uint_as_float(__float_as_uint(f) | ((code & 0x80u) << 24));
}
// four codes of a word -> four bfloat16 numbers
__device__ __forceinline__ void code_bf16(uint32_t w, const CodeBits& b, uint32_t& lo, uint32_t& hi) {
    const uint32_t v0 = __float_as_uint(code_value(w & 0xFFu, b)), v1 = __float_as_uint(code_value((w >> 8) & 0xFFu, b));
    const uint32_t v2 = __float_as_uint(code_value((w >> 16) & 0xFFu, b)), v3 = __float_as_uint(code_value(w >> 24, b));
    lo = __builtin_amdgcn_perm(v1, v0, 0x07060302u);
    hi = __builtin_amdgcn_perm(v3, v2, 0x07060302u);
}

// ---- operands laid out for the tile ---------------------------------------------------------

// Up to five operands are laid out by 256 lanes a workgroup: those from `first` on belong to a job.
enum { LAY_CODES = 0, LAY_BF16 = 1, LAY_TRANSPOSED = 2 };
struct LayJob {
    const uint8_t* src;      // [R, K] codes
    uint8_t* dst;
    int64_t R;
    int64_t ld;              // bytes of a row of dst
    int32_t K;
    int32_t wide;            // LAY_TRANSPOSED: R rounded up to 8: columns of dst, zeros from R on
    int32_t tiles_k;         // LAY_TRANSPOSED: tiles along k
    int32_t kind;
    uint32_t first;
    CodeBits bits;
};
struct LayJobs { LayJob job[5]; int32_t n; };

// rows of codes or of bfloat16 numbers, zeros behind K: 16 bytes of output a lane
template <bool BF16> __device__ __forceinline__ void lay_rows(const LayJob& p, int64_t block) {
    constexpr int PER = BF16 ? 8 : 16;
    const uint32_t per_row = (uint32_t)(p.ld / 16), i = (uint32_t)block * 256 + threadIdx.x;   // fewer than 2^30 pieces (lay_fits)
    if (i >= (uint32_t)p.R * per_row) return;
    const uint32_t r = i / per_row;
    const int k = (int)(i - r * per_row) * PER;
    const uint8_t* s = p.src + (int64_t)r * p.K + k;
    uint32_t w[PER / 4];
    if (k + PER <= p.K) {
        typedef uint32_t words __attribute__((ext_vector_type(PER / 4), aligned(1)));
        const words x = *(const words*)s;
#pragma unroll
        for (int j = 0; j < PER / 4; ++j) w[j] = x[j];
    } else {
#pragma unroll
        for (int j = 0; j < PER / 4; ++j) w[j] = 0;
#pragma unroll
        for (int j = 0; j < PER; ++j)
            if (k + j < p.K) w[j / 4] |= (uint32_t)s[j] << (8 * (j % 4));
    }
    i32x4 o;
    if constexpr (BF16) {
        uint32_t lo, hi;
        code_bf16(w[0], p.bits, lo, hi); o[0] = (int32_t)lo; o[1] = (int32_t)hi;
        code_bf16(w[1], p.bits, lo, hi); o[2] = (int32_t)lo; o[3] = (int32_t)hi;
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j) o[j] = (int32_t)w[j];
    }
    *(i32x4*)(p.dst + (int64_t)r * p.ld + (i - r * per_row) * 16) = o;
}

// dst [K][ld] bfloat16: 64 rows of 128 codes through LDS.  A lane reads four neighbouring codes of eight rows and writes four pieces of 16 bytes,
// eight lanes side by side; rows of 33 words put the words that a wave reads at a time into 64 different banks.
constexpr int kLayK = 128;
constexpr int kLayRow = kLayK / 4 + 1, kLayWords = 64 * kLayRow;
__device__ __forceinline__ void lay_transposed(const LayJob& p, int64_t block, uint32_t* t) {
    const int64_t r0 = block / p.tiles_k * 64;
    const int k0 = (int)(block % p.tiles_k) * kLayK;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const int i = h * 256 + threadIdx.x, r = i / 8, c = i % 8, k = k0 + c * 16;
        u32x4 w = {0, 0, 0, 0};
        if (r0 + r < p.R && k < p.K) {
            const uint8_t* s = p.src + (r0 + r) * p.K + k;
            if (k + 16 <= p.K) {
                typedef uint32_t words __attribute__((ext_vector_type(4), aligned(1)));
                w = *(const words*)s;
            } else {
#pragma unroll
                for (int j = 0; j < 16; ++j)
                    if (k + j < p.K) w[j / 4] |= (uint32_t)s[j] << (8 * (j % 4));
            }
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) t[r * kLayRow + c * 4 + j] = w[j];
    }
    __syncthreads();
    const int r = threadIdx.x % 8 * 8, kw = threadIdx.x / 8;
    if (r0 + r >= p.wide) return;
    uint32_t w[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) w[j] = t[(r + j) * kLayRow + kw];
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        const int k = k0 + kw * 4 + q;
        if (k >= p.K) return;
        i32x4 o;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const uint32_t a = __float_as_uint(code_value((w[2 * j] >> (8 * q)) & 0xFFu, p.bits));
            const uint32_t b = __float_as_uint(code_value((w[2 * j + 1] >> (8 * q)) & 0xFFu, p.bits));
            o[j] = (int32_t)__builtin_amdgcn_perm(b, a, 0x07060302u);
        }
        *(i32x4*)(p.dst + k * p.ld + (r0 + r) * 2) = o;
    }
}

// what workgroup `at` of the jobs does; `t`: kLayWords words of LDS
__device__ __forceinline__ void lay_block(const LayJobs& jobs, uint32_t at, uint32_t* t) {
    int j = 0;
    while (j + 1 < jobs.n && at >= jobs.job[j + 1].first) ++j;
    const LayJob& p = jobs.job[j];
    const int64_t block = at - p.first;
    if (p.kind == LAY_CODES) lay_rows<false>(p, block);
    else if (p.kind == LAY_BF16) lay_rows<true>(p, block);
    else lay_transposed(p, block, t);
}

// column sums that a launch of the gradient products makes beside them: out[n] = sum over `parts` rows of part[row][n], n < cols
struct SideSums { const float* part; float* out; int32_t parts, cols; };

enum { EPI_FORWARD = 0, EPI_BACKWARD = 1 };
// One launch of one product or two: workgroups below `blocks` belong to the first, from `all` on to the column sums; of the gradient of the
// sums: from `all` on to the operands that the gradient products read.
template <int EPI> struct DenseArgs { GemmParams g[2]; int32_t blocks, all; SideSums side; };
template <> struct DenseArgs<EPI_BACKWARD> { GemmParams g[1]; int32_t all; LayJobs side; };

// 16 columns a workgroup, THREADS / 16 lanes a column, which take its rows in turn, then their sums in a fixed order
template <int THREADS> __device__ __forceinline__ void side_sums(const SideSums& q, int block, float* lds) {
    constexpr int LANES = THREADS / 16;
    const int c = threadIdx.x & 15, n = block * 16 + c;
    float s = 0.0f;
    if (n < q.cols) {
        int r = threadIdx.x / 16;
        for (; r + 3 * LANES < q.parts; r += 4 * LANES) {
            float v[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) v[k] = q.part[(int64_t)(r + k * LANES) * q.cols + n];
            s += (v[0] + v[1]) + (v[2] + v[3]);
        }
        for (; r < q.parts; r += LANES) s += q.part[(int64_t)r * q.cols + n];
    }
    s += __shfl_xor(s, 16);
    s += __shfl_xor(s, 32);
    if ((threadIdx.x & 48) == 0) lds[threadIdx.x / 64 * 16 + c] = s;
    __syncthreads();
    if (threadIdx.x >= 16 || n >= q.cols) return;
    s = 0.0f;
#pragma unroll
    for (int w = 0; w < THREADS / 64; ++w) s += lds[w * 16 + c];
    q.out[n] = s;
}

__device__ __forceinline__ int up_to_8(int x) { return (x + 7) & ~7; }

// a lane's V columns: how many of them there are and their bias
template <bool GATED, int V> struct Columns { int n, cnt; float b[V], bu[V]; };
template <bool GATED, int V> __device__ __forceinline__ Columns<GATED, V> columns_of(const EpiParams& e, int n) {
    Columns<GATED, V> c;
    c.n = n;
    c.cnt = e.N - n;
#pragma unroll
    for (int j = 0; j < V; ++j) c.b[j] = c.bu[j] = 0.0f;
    if (e.bias && c.cnt > 0) {
        load_some<V>(e.bias + n, c.cnt, c.b);
        if (GATED) load_some<V>(e.bias + e.N + n, c.cnt, c.bu);
    }
    return c;
}

// Sums of one output's V columns -> Y.  z: the sums (gated: the gate's), u: the second half's, r: the residual's values if there is one.
template <bool GATED, bool INSIDE, int ACT, int V>
__device__ __forceinline__ void finish_forward(const EpiParams& e, const Columns<GATED, V>& c, uint64_t base, int m, const At& i, float (&z)[V], float (&u)[V],
                                               const float (&r)[V]) {
    if (!INSIDE && (m >= e.M || c.cnt <= 0)) return;
    const int cnt = INSIDE ? V : c.cnt;
#pragma unroll
    for (int j = 0; j < V; ++j) {
        if (j == 4) __builtin_amdgcn_sched_barrier(0);   // four at a time: more would only cost registers
        z[j] = act_value<ACT>(fmaf(z[j], e.scale, c.b[j]));
        if (GATED) z[j] *= fmaf(u[j], e.scale, c.bu[j]);
    }
    if (e.drop.on) {
        bool keep[V];
        drop_keeps<V>((uint64_t)i.u + i.o, base, e.drop, (e.N & 3) == 0, keep);
#pragma unroll
        for (int j = 0; j < V; ++j) z[j] = keep[j] ? z[j] * e.drop.keep_scale : 0.0f;
    }
    if (e.R) {
#pragma unroll
        for (int j = 0; j < V; ++j) z[j] += r[j];
    }
    if (e.y_type == LBA_F32) store_some<V>(at((float*)e.Y, i), cnt, z, e.fmt);
    else if (e.y_type == LBA_BF16) store_some<V>(at((bf16_t*)e.Y, i), cnt, z, e.fmt);
    else store_some<V>(at((uint8_t*)e.Y, i), cnt, z, e.fmt);
}
// what finish_forward adds, read at once
template <int V> __device__ __forceinline__ void load_extra(const EpiParams& e, int m, int n, float (&r)[V]) {
#pragma unroll
    for (int j = 0; j < V; ++j) r[j] = 0.0f;
    if (!e.R || m >= e.M || n >= e.N) return;
    if (e.r_type == LBA_F32) load_some<V>((const float*)e.R + (int64_t)m * e.N + n, e.N - n, r);
    else load_some<V>((const bf16_t*)e.R + (int64_t)m * e.N + n, e.N - n, r);
}

// Sums of one output's V columns -> the gradients of the sums, in z (and u); g: the output's gradient.
template <bool GATED, bool INSIDE, int ACT, int V>
__device__ __forceinline__ void finish_backward(const EpiParams& e, const Columns<GATED, V>& c, uint64_t base, int m, const At& i, float (&z)[V], float (&u)[V],
                                                const float (&g)[V]) {
    bool keep[V];
#pragma unroll
    for (int j = 0; j < V; ++j) keep[j] = true;
    if (e.drop.on) drop_keeps<V>((uint64_t)i.u + i.o, base, e.drop, (e.N & 3) == 0, keep);
#pragma unroll
    for (int j = 0; j < V; ++j) {
        if (j == 4) __builtin_amdgcn_sched_barrier(0);
        const bool on = (INSIDE || (m < e.M && j < c.cnt)) && keep[j];               // a dropped element's sums do not matter
        float value, slope;
        act_both<ACT>(fmaf(z[j], e.scale, c.b[j]), value, slope);
        const float d = g[j] * e.drop.keep_scale;                                    // 1 where nothing is dropped
        z[j] = on ? (GATED ? d * fmaf(u[j], e.scale, c.bu[j]) * slope : d * slope) : 0.0f;
        if (GATED) u[j] = on ? d * value : 0.0f;
    }
}

// eight values -> bfloat16: rounded to nearest, or (`piece` 0, 1, 2) the piece of float32 values that three pieces add up to exactly
// (truncate, subtract, truncate, subtract)
typedef uint16_t u16x8 __attribute__((ext_vector_type(8)));
__device__ __forceinline__ u16x8 eight_rounded(const float (&d)[8]) {
    u16x8 w;
#pragma unroll
    for (int j = 0; j < 8; ++j) w[j] = __builtin_bit_cast(uint16_t, (bf16_t)d[j]);
    return w;
}
__device__ __forceinline__ void eight_pieces(const float (&d)[8], u16x8 (&w)[3]) {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const uint32_t hi = __float_as_uint(d[j]) & 0xFFFF0000u;
        const float r1 = d[j] - __uint_as_float(hi);
        const uint32_t mid = __float_as_uint(r1) & 0xFFFF0000u;
        const float r2 = r1 - __uint_as_float(mid);
        w[0][j] = (uint16_t)(hi >> 16);
        w[1][j] = (uint16_t)(mid >> 16);
        w[2][j] = (uint16_t)(__float_as_uint(r2) >> 16);
    }
}
// Stores eight neighbouring values of the gradient matrix (16-byte aligned), or of its transpose.  Where the caller's gradients are bfloat16 the
// matrix is rounded to bfloat16 as well, each element for itself, so that its products are one pass of the matrix cores each: dA and dB of
// 4096 x (2 x 4096) x 1024 gated come out 2.35e-3 of their norm off, and 1.66e-3 is what their own rounding to bfloat16 leaves.  A second piece
// would take that away and twice the time of the two products, 117 us of that pass's 233.  Float32 gradients lose nothing.
__device__ __forceinline__ void store_eight(bf16_t* to, const At& i, int pieces, int64_t piece, const float (&d)[8]) {
    if (pieces == 1) {
        *(u16x8*)at(to, i) = eight_rounded(d);
        return;
    }
    u16x8 w[3];
    eight_pieces(d, w);
#pragma unroll
    for (int q = 0; q < 3; ++q) *(u16x8*)at(to + q * piece, i) = w[q];
}

// Which slice and tile a workgroup takes: consecutive workgroups go to the eight dies in turn, so that a die gets a contiguous run, of one
// slice before the next: the columns of a slice are read by the dies that have it.  A run goes down eight tiles of m before it moves on in n:
// both operands of a run are shared in the die's L2.
__device__ __forceinline__ void tile_of(int gx, int gy, int slices, int id, int& slice, int& tm, int& tn) {
    const int tiles = gx * gy, total = slices > 1 ? tiles * slices : tiles, per = total / 8, rem = total % 8, die = id % 8, local = id / 8;
    int t = die * per + (die < rem ? die : rem) + local;
    slice = slices > 1 ? t / tiles : 0;
    t -= slice * tiles;
    const int wide = 8 * gy, group = t / wide, first = group * 8, in = t % wide;
    const int rows = gx - first < 8 ? gx - first : 8;
    tm = first + in % rows;
    tn = in / rows;
}

__device__ const uint32_t lba_zero_piece[4] = {0, 0, 0, 0};

// what the rows hold: E4M3 codes, codes of at most 4 exponent bits that become FP16 numbers, or bfloat16 numbers
enum { ELEM_E4M3 = 0, ELEM_F16 = 1, ELEM_BF16 = 2 };

// eight codes -> the matrix core's eight 16-bit operands
template <int ELEM> __device__ __forceinline__ i32x4 eight_codes(uint32_t w0, uint32_t w1, int shift, uint32_t keep) {
    i32x4 v;
    if constexpr (ELEM == ELEM_E4M3) {
        v[0] = __builtin_bit_cast(int32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w0, 1.0f, false));
        v[1] = __builtin_bit_cast(int32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w0, 1.0f, true));
        v[2] = __builtin_bit_cast(int32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w1, 1.0f, false));
        v[3] = __builtin_bit_cast(int32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w1, 1.0f, true));
    } else {
        // A code in the high byte of a half, shifted down with its sign, is the FP16 number but for the sign's copies and what lies below:
        // `keep` takes those out.  The bytes of a word come in the order 1, 3, 0, 2, for both operands.
        typedef int16_t i16x2 __attribute__((ext_vector_type(2)));
        const i16x2 s2 = {(int16_t)shift, (int16_t)shift};
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const uint32_t w = i ? w1 : w0;
            v[2 * i] = (int32_t)(__builtin_bit_cast(uint32_t, __builtin_bit_cast(i16x2, w) >> s2) & keep);
            v[2 * i + 1] = (int32_t)(__builtin_bit_cast(uint32_t, __builtin_bit_cast(i16x2, w << 8) >> s2) & keep);
        }
    }
    return v;
}
template <int ELEM> __device__ __forceinline__ f32x4 product_16x16x32(i32x4 b, i32x4 a, f32x4 c) {
    if constexpr (ELEM == ELEM_F16) return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8_t, b), __builtin_bit_cast(f16x8_t, a), c, 0, 0, 0);
    else return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, b), __builtin_bit_cast(bf16x8_t, a), c, 0, 0, 0);
}

// WM x WN waves of FM x FN fragments of 16 x 16, NST buffers of a step.  NA == 3: A comes in three pieces, whose products with a step of B are
// made together: a step is 64 bytes of a row, and B's rows and fragments are read once for the three.
template <int ELEM, int WM, int WN, int FM, int FN, int NST, int NA, bool GATED, int EPI>
__global__ __launch_bounds__(WM * WN * 64, (FM == 2 ? 4 : 2) / (NST > 2 ? 2 : 1)) void dense_kernel(DenseArgs<EPI> both) {
    bool second = false;
    int id = (int)blockIdx.x;
    if constexpr (EPI == EPI_FORWARD) {
        second = id >= both.blocks;
        if (second) id -= both.blocks;
    }
    const GemmParams& p = both.g[second];
    constexpr int THREADS = WM * WN * 64, BM = WM * FM * 16, BN = WN * FN * 16;
    constexpr int CH16 = NA == 3 ? 4 : 8, ROW = CH16 * 16;               // sixteens of bytes of a row in a step, bytes
    constexpr int LA = NA * BM * CH16 / THREADS, LB = BN * CH16 / THREADS;           // sixteens that a lane stages for a step
    static_assert(NA * BM * CH16 % THREADS == 0 && BN * CH16 % THREADS == 0 && THREADS / CH16 <= BM && (!GATED || FN % 2 == 0), "tile");
    static_assert(NA == 1 || (NA == 3 && ELEM == ELEM_BF16 && !GATED && NST == 2), "three pieces");
    __shared__ __attribute__((aligned(16))) uint8_t lds[NST][(NA * BM + BN) * ROW];
    if constexpr (EPI == EPI_BACKWARD) {
        static_assert(THREADS == 256 && sizeof(lds) >= kLayWords * 4, "jobs beside the tile");
        if ((int)blockIdx.x >= both.all) {
            lay_block(both.side, blockIdx.x - both.all, (uint32_t*)&lds[0][0]);
            return;
        }
    } else if constexpr (ELEM == ELEM_BF16 && !GATED) {
        if ((int)blockIdx.x >= both.all) {
            side_sums<THREADS>(both.side, (int)blockIdx.x - both.all, (float*)&lds[0][0]);
            return;
        }
    }
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid / 64);
    const int wm = wave / WN, wn = wave % WN;
    int slice, tm, tn;
    tile_of(p.gx, p.gy, p.slices, id, slice, tm, tn);
    const int m0 = tm * BM, n0 = tn * (GATED ? BN / 2 : BN);

    // staging: lane's rows and its piece of each
    const int piece = (tid & (CH16 - 1)) ^ ((tid / CH16 / 2) & (CH16 - 1));
    const uint8_t* src[LA + LB];
#pragma unroll
    for (int i = 0; i < LA; ++i) {
        const int t = tid / CH16 + i * (THREADS / CH16);
        int r = m0 + t % BM;
        r = r < p.rows_a ? r : p.rows_a - 1;
        src[i] = p.A + r * p.lda + t / BM * p.a_piece + piece * 16;
    }
#pragma unroll
    for (int i = 0; i < LB; ++i) {
        const int t = tid / CH16 + i * (THREADS / CH16);
        int r;
        if (GATED) {                                     // fragments alternate between the halves, so that a wave has both of a column
            const int n = n0 + (t / 32) * 16 + t % 16;
            r = (n < p.half ? n : p.half - 1) + ((t / 16) % 2) * p.half;
        } else {
            r = n0 + t;
            r = r < p.rows_b ? r : p.rows_b - 1;
        }
        src[LA + i] = p.B + r * p.ldb + piece * 16;
    }
#pragma unroll
    for (int i = 0; i < LA + LB; ++i) asm volatile("" : "+v"(src[i]));               // one address a load, not a sum of parts at every step
    // what the loop reads of the parameters, once
    const int chunks = p.chunks, shift_a = p.shift_a, shift_b = p.shift_b;
    const uint32_t keep_a = p.keep_a, keep_b = p.keep_b;
    const int first = slice * p.per_slice;
    const int last = p.slices > 1 ? (first + p.per_slice < p.steps ? first + p.per_slice : p.steps) : p.steps;
    int at_step = first;                                 // the step that is staged next, and its place in the rows
    int64_t at_byte = (int64_t)first * ROW;
    auto stage = [&](int buf) {
        auto to_lds = [&](int i, const uint8_t* g) {
            uint8_t* l = &lds[buf][((i < LA ? i : i - LA) * THREADS + wave * 64) * 16 + (i < LA ? 0 : NA * BM * ROW)];
            __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) uint32_t*)g,
                                             (__attribute__((address_space(3))) uint32_t*)l, 16, 0, 0);
        };
        if (at_step * CH16 + CH16 <= chunks) {
#pragma unroll
            for (int i = 0; i < LA + LB; ++i) to_lds(i, src[i] + at_byte);
        } else {                                         // the rows end inside this step
            const bool in = at_step * CH16 + piece < chunks;
#pragma unroll
            for (int i = 0; i < LA + LB; ++i) to_lds(i, in ? src[i] + at_byte : (const uint8_t*)lba_zero_piece);
        }
        at_byte += ROW;
        ++at_step;
    };

    f32x4 acc[FM][FN];
#pragma unroll
    for (int i = 0; i < FM; ++i)
#pragma unroll
        for (int j = 0; j < FN; ++j) acc[i][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};

    const int place = ((lane / 16) ^ (((lane & 15) >> 1) & (CH16 - 1))) * 16 + (lane & 15) * ROW;
    const int flip = (place & 64) ? -64 : 64;            // the second piece of a row is 64 bytes on, modulo the row
#pragma unroll
    for (int i = 0; i < NST - 1; ++i)
        if (first + i < last) stage(i);
    i32x4 ra[2][FM], rb[2][FN];
    auto read = [&](int h, int buf) {
        const uint8_t* la = &lds[buf][wm * FM * 16 * ROW + place];
        const uint8_t* lb = &lds[buf][NA * BM * ROW + wn * FN * 16 * ROW + place];
#pragma unroll
        for (int j = 0; j < FN; ++j) rb[h][j] = *(const i32x4*)(lb + j * 16 * ROW + h * flip);
#pragma unroll
        for (int i = 0; i < FM; ++i) ra[h][i] = *(const i32x4*)(la + i * 16 * ROW + h * flip);
    };
    auto multiply = [&](int h) {
        if constexpr (ELEM == ELEM_BF16) {
#pragma unroll
            for (int i = 0; i < FM; ++i)
#pragma unroll
                for (int j = 0; j < FN; ++j) acc[i][j] = product_16x16x32<ELEM>(rb[h][j], ra[h][i], acc[i][j]);
        } else {
#pragma unroll
            for (int s = 0; s < 2; ++s) {
                i32x4 fb[FN];
#pragma unroll
                for (int j = 0; j < FN; ++j) fb[j] = eight_codes<ELEM>((uint32_t)rb[h][j][2 * s], (uint32_t)rb[h][j][2 * s + 1], shift_b, keep_b);
#pragma unroll
                for (int i = 0; i < FM; ++i) {
                    const i32x4 fa = eight_codes<ELEM>((uint32_t)ra[h][i][2 * s], (uint32_t)ra[h][i][2 * s + 1], shift_a, keep_a);
#pragma unroll
                    for (int j = 0; j < FN; ++j) acc[i][j] = product_16x16x32<ELEM>(fb[j], fa, acc[i][j]);
                }
            }
        }
    };
    int buf = 0;
#pragma unroll 1
    for (int step = first; step < last; ++step) {
        // This step's loads have to be done, those of the NST - 2 steps after it may be under way.  A step is LA + LB loads a wave or more,
        // and loads end in order.  What was read of the step before is in registers: its buffer is staged next.
        if (NST > 3 && step + 2 < last) asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(2 * (LA + LB)) : "memory");
        else if (NST > 2 && step + 1 < last) asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(LA + LB) : "memory");
        else asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
        __builtin_amdgcn_s_barrier();                    // every wave's loads of this step are done, and the step before is read
        asm volatile("" ::: "memory");
        if constexpr (NA == 3) {
            read(0, buf);
            __builtin_amdgcn_sched_barrier(0);
            if (step + 1 < last) stage(buf ^ 1);
            const uint8_t* la = &lds[buf][wm * FM * 16 * ROW + place];
#pragma unroll
            for (int q = 0; q < 3; ++q) {                // the next piece's fragments are read before this one's products
                if (q < 2) {
#pragma unroll
                    for (int i = 0; i < FM; ++i) ra[(q + 1) & 1][i] = *(const i32x4*)(la + ((q + 1) * BM + i * 16) * ROW);
                    __builtin_amdgcn_sched_barrier(0);
                }
#pragma unroll
                for (int i = 0; i < FM; ++i)
#pragma unroll
                    for (int j = 0; j < FN; ++j) acc[i][j] = product_16x16x32<ELEM>(rb[0][j], ra[q & 1][i], acc[i][j]);
            }
            buf ^= 1;
            continue;
        }
        // the first half's fragments are read before the next step's loads are issued, the second half's before the first half's products
        read(0, buf);
        __builtin_amdgcn_sched_barrier(0);
        if (step + NST - 1 < last) stage(buf == 0 ? NST - 1 : buf - 1);
        if (FM < 6) {                                    // (large tiles have no registers for both halves)
            read(1, buf);
            __builtin_amdgcn_sched_barrier(0);
            multiply(0);
        } else {
            multiply(0);
            read(1, buf);
        }
        multiply(1);
        buf = buf == NST - 1 ? 0 : buf + 1;
    }
    __syncthreads();

    if (p.slices > 1) {                                  // one slice of the sum: raw, for the launch that adds the slices
        const int mr = m0 + wm * FM * 16 + (lane & 15), nr = n0 + (GATED ? wn * FN * 8 : wn * FN * 16) + (lane / 16) * 4;
        float* out = p.split + (int64_t)slice * p.e.M * p.rows_b;
        const CodeFmt none = {};
#pragma unroll
        for (int i = 0; i < FM; ++i)
#pragma unroll
            for (int j = 0; j < FN; ++j) {
                const int m = mr + i * 16, n = GATED ? nr + (j / 2) * 16 : nr + j * 16;
                const int lim = GATED ? p.half : p.rows_b;
                float z[4];
#pragma unroll
                for (int k = 0; k < 4; ++k) z[k] = acc[i][j][k];
                if (m < p.e.M && n < lim) store_some<4>(out + (int64_t)m * p.rows_b + (GATED && (j & 1) ? p.half : 0) + n, lim - n, z, none);
            }
        return;
    }
    // The sums go through LDS, at most 64 rows of a wave at a time, so that a lane has eight neighbouring columns and neighbouring lanes the next
    // ones: a wave works on its own part, without barriers.  Place of the four columns c of row r: (c / 4) ^ (r % CH), which spreads a
    // column over the banks.
    typedef PartShape<FN, GATED> Part;
    constexpr int EH = FM == 8 ? 4 : FM == 6 ? 3 : FM, CH = Part::CH, LPR = Part::LPR;               // rows of fragments, fours of a row, lanes of a row
    constexpr int RPP = Part::RPP, PASSES = EH * 16 / RPP;     // rows of a pass, passes
    static_assert(PASSES >= 1 && FM / EH <= 2 && FM % EH == 0 && sizeof(lds) >= (size_t)WM * WN * EH * 16 * CH * 16, "epilogue");
    float* mine = (float*)&lds[0][0] + wave * (EH * 16 * CH * 4);
    const EpiParams e = p.e;
    const uint64_t base = e.drop.on ? drop_base(e.drop) : 0;
    const int oct = lane % LPR;
    const int cz = GATED ? oct / 2 * 8 + oct % 2 * 2 : oct * 2;                      // the first of its two places in the row of sums
    const int nw = n0 + wn * (GATED ? FN * 8 : FN * 16), ncol = nw + oct * 8;
    const Columns<GATED, 8> cols = columns_of<GATED, 8>(e, ncol);
    const void* extra = EPI == EPI_FORWARD ? e.R : e.G;
    const int extra_type = EPI == EPI_FORWARD ? e.r_type : e.g_type;
    float sz[8], su[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) sz[k] = su[k] = 0.0f;
    auto get = [&](int r, int c, float (&v)[8]) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const f32x4 x = *(const f32x4*)(mine + (r * CH + ((c + h) ^ (r % CH))) * 4);
#pragma unroll
            for (int k = 0; k < 4; ++k) v[4 * h + k] = x[k];
        }
    };
    auto put = [&](int r, int c, const float (&v)[8]) {
#pragma unroll
        for (int h = 0; h < 2; ++h) *(f32x4*)(mine + (r * CH + ((c + h) ^ (r % CH))) * 4) = f32x4{v[4 * h], v[4 * h + 1], v[4 * h + 2], v[4 * h + 3]};
    };
#pragma unroll 1
    for (int h = 0; h < FM / EH; ++h) {                  // one copy of the code for both halves
        const int mh = m0 + (wm * FM + h * EH) * 16;
        int l = lane;
        asm volatile("" : "+v"(l));                      // addresses are made anew for each half: kept, they would cost the passes' registers
        const int row_in = l / LPR;
#pragma unroll
        for (int i = 0; i < EH; ++i)
#pragma unroll
            for (int j = 0; j < FN; ++j) {
                const int r = i * 16 + (l & 15), c = j * 4 + l / 16;
                *(f32x4*)(mine + (r * CH + (c ^ (r % CH))) * 4) = acc[i][j];
                // the second half's sums move into the first's registers, which are free while the passes run
                if (FM > EH) acc[i][j] = acc[FM > EH ? EH + i : i][j];
            }
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
        __builtin_amdgcn_wave_barrier();
        // one pass: a lane's row r (m of the output, at index i; ip in the gradient matrix) with the residual's or gradient's values x
        auto pass = [&](auto inside, auto act, int r, const At& i, const At& ip, const float (&x)[8]) {
            constexpr bool INSIDE = decltype(inside)::value != 0;
            const int m = mh + r;
            float z[8], u[8];
            get(r, cz, z);
            if (GATED) get(r, cz + 4, u);
            if constexpr (EPI == EPI_FORWARD) {
                finish_forward<GATED, INSIDE, decltype(act)::value, 8>(e, cols, base, m, i, z, u, x);
            } else {
                finish_backward<GATED, INSIDE, decltype(act)::value, 8>(e, cols, base, m, i, z, u, x);
                if (e.P && (INSIDE || (m < e.M && ncol < e.wide))) {              // wide and ncol are multiples of 8; zeros up to `wide`
                    store_eight(e.P, ip, e.pieces, e.p_piece, z);
                    if (GATED) store_eight(e.P + e.wide, ip, e.pieces, e.p_piece, u);
                }
                put(r, cz, z);
                if (GATED) put(r, cz + 4, u);
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    sz[k] += z[k];
                    if (GATED) su[k] += u[k];
                }
            }
        };
        const int64_t u0 = (int64_t)mh * e.N + nw, up = mh * e.ldp + nw;
        constexpr bool LONG = ELEM == ELEM_BF16 && !GATED && EPI == EPI_FORWARD;     // the gradients of the operands
        auto out_at = [&](int g) { return lane_at<FN, GATED, LONG>(u0, e.N, l, g); };
        auto grad_at = [&](int g) { return lane_at<FN, GATED, false>(up, e.ldp, l, g); };
        // Wholly inside: the next pass's residuals or gradients are under way, as they are, before this one's results are stored: a load
        // that follows stores waits for them too.
        auto passes = [&](auto act) {
            u32x4 raw[2][2];
            auto fetch = [&](int g, u32x4 (&w)[2]) {
                const At i = out_at(g);
                if (extra && extra_type == LBA_F32) {
                    w[0] = *(const u32x4_any*)at((const float*)extra, i);
                    w[1] = *(const u32x4_any*)(at((const float*)extra, i) + 4);
                } else if (extra) {
                    w[0] = *(const u32x4_any*)at((const bf16_t*)extra, i);
                }
            };
            auto work = [&](int g, const u32x4 (&w)[2]) {
                float x[8];
#pragma unroll
                for (int k = 0; k < 8; ++k) x[k] = 0.0f;
                if (extra && extra_type == LBA_F32) {
#pragma unroll
                    for (int k = 0; k < 8; ++k) x[k] = __uint_as_float(w[k / 4][k % 4]);
                } else if (extra) {
#pragma unroll
                    for (int k = 0; k < 8; ++k) x[k] = __uint_as_float(k % 2 ? w[0][k / 2] & 0xFFFF0000u : w[0][k / 2] << 16);
                }
                pass(Known<1>{}, act, g * RPP + row_in, out_at(g), grad_at(g), x);
            };
            fetch(0, raw[0]);
#pragma unroll 1
            for (int g = 0; g < PASSES; g += 2) {
                if (g + 1 < PASSES) fetch(g + 1, raw[1]);
                work(g, raw[0]);
                if (g + 1 < PASSES) {
                    if (g + 2 < PASSES) fetch(g + 2, raw[0]);
                    work(g + 1, raw[1]);
                }
            }
        };
        // The last rows and columns: what is beyond them reads as the last one and is not stored.
        auto edge_passes = [&](auto act) {
#pragma unroll 1
            for (int g = 0; g < PASSES; ++g) {
                const int r = g * RPP + row_in, m = mh + r;
                float x[8];
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    const int64_t i = (int64_t)(m < e.M ? m : e.M - 1) * e.N + (ncol + k < e.N ? ncol + k : e.N - 1);
                    x[k] = !extra ? 0.0f : extra_type == LBA_F32 ? ((const float*)extra)[i] : (float)((const bf16_t*)extra)[i];
                }
                pass(Known<0>{}, act, r, out_at(g), grad_at(g), x);
            }
        };
        const bool inside = mh + EH * 16 <= e.M && nw + LPR * 8 <= e.N;
        const bool some = EPI == EPI_BACKWARD ? mh < up_to_8(e.M) && nw < e.wide : mh < e.M && nw < e.N;
        with_act(e.act, [&](auto act) {
            if (inside) passes(act);
            else if (some) edge_passes(act);
        });
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
        __builtin_amdgcn_wave_barrier();
        if constexpr (EPI == EPI_BACKWARD) {
            if (e.PT && mh < up_to_8(e.M) && nw < e.N) {        // the transposed copy: eight rows of one column a lane
                constexpr int LM = EH * 2, NPP = 64 / LM;                            // lanes along m, columns of a pass
                const int r0 = (lane % LM) * 8, m = mh + r0;
#pragma unroll 1
                for (int c0 = 0; c0 < CH * 4; c0 += NPP) {
                    const int c = c0 + lane / LM;
                    const int n = nw + (GATED ? c / 32 * 16 + c % 16 : c);
                    const int half = GATED ? c / 16 % 2 : 0;
                    float d[8];
                    if (lane < LM * NPP && c < CH * 4 && n < e.N && m < up_to_8(e.M)) {          // m is a multiple of 8: zeros beyond M are part of the copy
#pragma unroll
                        for (int k = 0; k < 8; ++k) d[k] = mine[((r0 + k) * CH + ((c / 4) ^ ((r0 + k) % CH))) * 4 + c % 4];
                        const At it = {((int64_t)half * e.N + n) * e.ldt + m, 0};
                        store_eight(e.PT, it, e.pieces, e.pt_piece, d);
                    }
                }
                __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
                __builtin_amdgcn_wave_barrier();
            }
        }
    }
    if constexpr (EPI == EPI_BACKWARD) {
        if (e.part) {                                    // column sums of the wave's rows: over the lanes that share a column
#pragma unroll
            for (int k = 0; k < 8; ++k) {
#pragma unroll
                for (int d = LPR; d < 64; d *= 2) {
                    sz[k] += __shfl_xor(sz[k], d);
                    if (GATED) su[k] += __shfl_xor(su[k], d);
                }
            }
            if (lane < LPR && ncol < e.N) {
                float* out = e.part + (int64_t)(tm * WM + wm) * (GATED ? 2 * e.N : e.N);
                store_some<8>(out + ncol, e.N - ncol, sz, e.fmt);
                if (GATED) store_some<8>(out + e.N + ncol, e.N - ncol, su, e.fmt);
            }
        }
    }
}

// Tiles: rows of outputs, columns of B, waves over m, lanes of a workgroup.  The deep ones have four buffers instead of two, for bfloat16 rows:
// their steps are shorter than the time a load takes where a CU has one workgroup (codes' are not: conversions fill them, and four buffers gained nothing).
enum { TILE_256 = 0, TILE_128 = 1, TILE_64 = 2, TILE_192 = 3, TILE_128_DEEP = 4, TILE_64_DEEP = 5, TILE_256_THREE = 6, TILE_128_THREE = 7, TILE_64_THREE = 8 };
struct TileShape { int bm, bn, wm, threads; };
inline TileShape tile_shape(int tile) {
    static const TileShape all[] = {{256, 256, 2, 512}, {128, 128, 2, 256}, {64, 64, 2, 256}, {192, 256, 2, 512}, {128, 128, 2, 256}, {64, 64, 2, 256},
                                    {256, 256, 2, 512}, {128, 128, 2, 256}, {64, 64, 2, 256}};
    return all[tile];
}

// A format as the kernels read it: how its codes become 16-bit operands, and the factor that is left (value = operand * factor).
struct ElemFmt { int elem, shift; uint32_t keep; float factor; };
inline ElemFmt make_elem(const lba_infmt& f, int elem) {
    const int bc = (1 << (f.exp_bits - 1)) - 1;
    ElemFmt e = {elem, f.man_bits - 2, (0x8000u | 0x7Fu << (10 - f.man_bits)) * 0x10001u, 0.0f};
    e.factor = __builtin_ldexpf(1.0f, elem == ELEM_F16 ? 15 - f.bias : bc - f.bias);
    return e;
}
// one kind for both operands of a product
inline int elem_of(const lba_infmt& a, const lba_infmt& b) {
    if (a.exp_bits == 4 && b.exp_bits == 4) return ELEM_E4M3;
    return a.exp_bits <= 4 && b.exp_bits <= 4 ? ELEM_F16 : ELEM_BF16;
}

// Few rows (at most kTokenRows): a pass over B (lba_dense_token.hip).  It and the tile, in us, operands in the last-level cache:
//                                   1 row          32             48             64
//   2304 x 768   E4M3               3.0 /  6.1     3.7 /  6.0     4.1 /  6.2     4.5 /  6.1
//   4096 x 4096  E4M3               5.2 / 10.1     8.3 / 11.8    10.3 / 11.3    12.2 / 12.0
//   4096 x 4096  M4E3               5.7 / 11.3     8.4 / 12.9    10.5 / 14.2    12.4 / 16.0
//   4096 x 4096  E5M2              12.3 / 27.6    17.7 / 25.7    22.2 / 26.1    27.2 / 26.6
//   2 x 4096 x 2048 E4M3, gated     4.9 / 10.8     6.5 / 10.4     7.6 / 10.5     8.8 / 10.4
//   8192 x 4096  E4M3               7.5 / 12.7    13.8 / 13.6    17.4 / 14.4    21.9 / 15.1
//   512 x 4608   E4M3               4.8 /  8.9     8.4 /  9.6    10.4 /  9.7    12.4 /  9.8
//   771 x 770    E4M3 (copied)      4.9 /  9.6     8.0 / 10.1     9.9 / 10.1    10.9 / 10.2
// 64 is where the two meet on most of them; from 32 rows on the tile is ahead on long rows of few or of very many columns.
constexpr int kTokenRows = 64;
struct TokenParams {
    const uint8_t* A;
    const uint8_t* B;
    int32_t M, K, rows_b, half;
    ElemFmt fa, fb;
    CodeBits ca, cb;         // ELEM_BF16
    EpiParams e;
};
void launch_dense_token(const TokenParams& p, int elem, bool gated, hipStream_t st);

// what runs beside: column sums (of a plain product of bfloat16 rows), or workgroups of jobs (of the gradient of the sums)
struct Beside { SideSums sums; LayJobs jobs; uint32_t job_blocks; };

// launches one or two products (b may be null) whose parameters are complete but for the grid, all in tiles of one shape; `side` may be null
int launch_dense_e4m3(const GemmParams& a, const GemmParams* b, const Beside* side, int tile, bool gated, int epi, hipStream_t st);
int launch_dense_f16(const GemmParams& a, const GemmParams* b, const Beside* side, int tile, bool gated, int epi, hipStream_t st);
int launch_dense_bf16(const GemmParams& a, const GemmParams* b, const Beside* side, int tile, bool gated, int epi, hipStream_t st);

inline int dense_grid(GemmParams& p, const TileShape& s, bool gated) {
    p.gx = (p.e.M + s.bm - 1) / s.bm;
    p.gy = gated ? (p.half + s.bn / 2 - 1) / (s.bn / 2) : (p.rows_b + s.bn - 1) / s.bn;
    return p.gx * p.gy * (p.slices > 1 ? p.slices : 1);
}

template <int ELEM> int launch_dense(const GemmParams& a, const GemmParams* b, const Beside* side, int tile, bool gated, int epi, hipStream_t st) {
    const TileShape s = tile_shape(tile);
    DenseArgs<EPI_FORWARD> fwd;
    DenseArgs<EPI_BACKWARD> bwd;
    dim3 grid;
    if (epi == EPI_FORWARD) {
        fwd.g[0] = a;
        fwd.g[1] = b ? *b : a;
        fwd.blocks = dense_grid(fwd.g[0], s, gated);
        fwd.all = fwd.blocks + (b ? dense_grid(fwd.g[1], s, gated) : 0);
        fwd.side = side ? side->sums : SideSums{};
        grid = dim3((unsigned)(fwd.all + (fwd.side.cols + 15) / 16));
    } else {
        bwd.g[0] = a;
        bwd.all = dense_grid(bwd.g[0], s, gated);
        bwd.side = side ? side->jobs : LayJobs{};
        grid = dim3((unsigned)bwd.all + (side ? side->job_blocks : 0u));
    }
    auto args = [&](auto e) -> auto& {
        if constexpr (decltype(e)::value == EPI_FORWARD) return fwd;
        else return bwd;
    };
#define LBA_DENSE(TILE, WM, WN, FM, FN, NST, NA, GATED, EPI) \
    if (tile == TILE && gated == GATED && epi == EPI) { \
        hipLaunchKernelGGL((dense_kernel<ELEM, WM, WN, FM, FN, NST, NA, GATED, EPI>), grid, dim3(WM * WN * 64), 0, st, args(Known<EPI>{})); \
        return LBA_OK; \
    }
#define LBA_DENSE_SMALL(GATED, EPI) LBA_DENSE(TILE_128, 2, 2, 4, 4, 2, 1, GATED, EPI) LBA_DENSE(TILE_64, 2, 2, 2, 2, 2, 1, GATED, EPI)
    LBA_DENSE_SMALL(false, EPI_FORWARD)
    LBA_DENSE_SMALL(true, EPI_FORWARD)
    LBA_DENSE(TILE_256, 2, 4, 8, 4, 2, 1, false, EPI_FORWARD)
    LBA_DENSE(TILE_256, 2, 4, 8, 4, 2, 1, true, EPI_FORWARD)
    LBA_DENSE_SMALL(false, EPI_BACKWARD)
    LBA_DENSE_SMALL(true, EPI_BACKWARD)
    if constexpr (ELEM == ELEM_BF16) {
        LBA_DENSE(TILE_128_DEEP, 2, 2, 4, 4, 4, 1, false, EPI_FORWARD)
        LBA_DENSE(TILE_64_DEEP, 2, 2, 2, 2, 4, 1, false, EPI_FORWARD)
        LBA_DENSE(TILE_256_THREE, 2, 4, 8, 4, 2, 3, false, EPI_FORWARD)
        LBA_DENSE(TILE_128_THREE, 2, 2, 4, 4, 2, 3, false, EPI_FORWARD)
        LBA_DENSE(TILE_64_THREE, 2, 2, 2, 2, 2, 3, false, EPI_FORWARD)
    } else {                                             // of codes: bfloat16 rows have no costs for it
        LBA_DENSE(TILE_192, 2, 4, 6, 4, 2, 1, false, EPI_FORWARD)
        LBA_DENSE(TILE_192, 2, 4, 6, 4, 2, 1, true, EPI_FORWARD)
    }
#undef LBA_DENSE_SMALL
#undef LBA_DENSE
    return LBA_ERR_UNSUPPORTED;                          // a tile that the plan must not choose here
}

}  // namespace lba
#endif

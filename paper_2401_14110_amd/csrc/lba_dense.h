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
// straight to LDS (16 bytes a lane, no registers in between) into one of two buffers while the matrix cores work on the other.
// A row of 128 bytes is 8 pieces of 16; piece c of row r stands at place c ^ (r / 2 % 8), so that the sixteen rows of a fragment
// read, 16 bytes each, fall on all 64 banks once.  An operand's pieces beyond the end of its rows are read from a zero page and
// rows beyond the last one repeat it: their outputs are not stored.
// Fragments: lane l holds row l % 16 and pieces l / 16 and l / 16 + 4 of the step, the same places of k for both operands, so it does
// not matter in which order the matrix core walks over them.  B is the first factor, so lane l ends up with output row l % 16 and
// four neighbouring columns 4 * (l / 16) ..: epilogues work on four columns at a time.
#ifndef LBA_DENSE_H_
#define LBA_DENSE_H_

#include "lba_layer_device.h"

namespace lba {

typedef int32_t i32x4 __attribute__((ext_vector_type(4)));
typedef int32_t i32x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
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
    bf16_t* P;               // [pieces][M][ldp]: N columns and zeros up to `wide`, gated: the second half's from `wide` on
    bf16_t* PT;              // [pieces][N or 2 N][ldt]
    int64_t ldp, ldt, p_piece, pt_piece;
    int32_t wide;            // N rounded up to 8
    float* part;             // [rows of partial sums][N or 2 N], or null
};

struct GemmParams {
    const uint8_t* A;
    const uint8_t* B;
    int64_t lda, ldb;        // bytes from row to row
    int64_t a_piece;         // bytes from piece to piece of A (a sum over pieces of A against the same B)
    int32_t pieces;
    int32_t rows_a, rows_b;
    int32_t half;            // gated: first row of B's second half
    int32_t chunks;          // 16-byte pieces of a row
    int32_t steps;           // steps of 128 bytes over all pieces of A
    int32_t gx, gy;          // tiles over m and n
    int32_t slices;          // the steps are cut into so many slices of `per_slice`, each of which stores its sums (split > 0)
    int32_t per_slice;
    float* split;            // [slices][M][N] raw sums, or null
    int32_t shift_a, shift_b;     // ELEM_F16: M - 2 of the operand's format
    uint32_t keep_a, keep_b;      // and the magnitude's places in both halves of a word
    EpiParams e;
};

__device__ __forceinline__ void load_typed4(const void* at, int type, int64_t i, int n, float (&v)[4]) {
    if (type == LBA_F32) load_some<4>((const float*)at + i, n, v);
    else load_some<4>((const bf16_t*)at + i, n, v);
}

// a lane's four columns: how many there are and their bias
template <bool GATED> struct Columns { int n, cnt; float b[4], bu[4]; };
template <bool GATED> __device__ __forceinline__ Columns<GATED> columns_of(const EpiParams& e, int n) {
    Columns<GATED> c;
    c.n = n;
    c.cnt = e.N - n;
#pragma unroll
    for (int j = 0; j < 4; ++j) c.b[j] = c.bu[j] = 0.0f;
    if (e.bias && c.cnt > 0) {
        load_some<4>(e.bias + n, c.cnt, c.b);
        if (GATED) load_some<4>(e.bias + e.N + n, c.cnt, c.bu);
    }
    return c;
}

// sums of one output's four columns -> Y.  z: the sums (gated: the gate's), u: the second half's, r: the residual's values if there is one
template <bool GATED> __device__ __forceinline__ void finish_forward(const EpiParams& e, const Columns<GATED>& c, uint64_t base, int m, float (&z)[4],
                                                                     float (&u)[4], const float (&r)[4]) {
    if (m >= e.M || c.cnt <= 0) return;
    const int64_t i = (int64_t)m * e.N + c.n;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        z[j] = fmaf(z[j], e.scale, c.b[j]);
        if (GATED) u[j] = fmaf(u[j], e.scale, c.bu[j]);
    }
    if (e.act != LBA_ACT_NONE) {
#pragma unroll
        for (int j = 0; j < 4; ++j) z[j] = act_value(z[j], e.act);
    }
    if (GATED) {
#pragma unroll
        for (int j = 0; j < 4; ++j) z[j] *= u[j];
    }
    if (e.drop.threshold) {
        float f[4];
        drop_factors<4>((uint64_t)i, base, e.drop.threshold, e.drop.keep_scale, f);
#pragma unroll
        for (int j = 0; j < 4; ++j) z[j] = f[j] != 0.0f ? z[j] * f[j] : 0.0f;
    }
    if (e.R) {
#pragma unroll
        for (int j = 0; j < 4; ++j) z[j] += r[j];
    }
    if (e.y_type == LBA_F32) store_some<4>((float*)e.Y + i, c.cnt, z, e.fmt);
    else if (e.y_type == LBA_BF16) store_some<4>((bf16_t*)e.Y + i, c.cnt, z, e.fmt);
    else store_some<4>((uint8_t*)e.Y + i, c.cnt, z, e.fmt);
}
// what finish_forward adds and finish_backward starts from
__device__ __forceinline__ void load_extra(const EpiParams& e, const void* at, int type, int m, int n, float (&r)[4]) {
#pragma unroll
    for (int j = 0; j < 4; ++j) r[j] = 0.0f;
    if (at && m < e.M && n < e.N) load_typed4(at, type, (int64_t)m * e.N + n, e.N - n, r);
}

// the pieces of a gradient: one, rounded to nearest, or three that add up to it exactly (truncate, subtract, truncate, subtract)
__device__ __forceinline__ void bf16_pieces(float d, int pieces, bf16_t (&p)[3]) {
    if (pieces == 1) { p[0] = p[1] = p[2] = (bf16_t)d; return; }
    const uint32_t hi = __float_as_uint(d) & 0xFFFF0000u;
    const float r1 = d - __uint_as_float(hi);
    const uint32_t mid = __float_as_uint(r1) & 0xFFFF0000u;
    const float r2 = r1 - __uint_as_float(mid);
    p[0] = __builtin_bit_cast(bf16_t, (uint16_t)(hi >> 16));
    p[1] = __builtin_bit_cast(bf16_t, (uint16_t)(mid >> 16));
    p[2] = __builtin_bit_cast(bf16_t, (uint16_t)(__float_as_uint(r2) >> 16));
}

// sums of one output's four columns -> the gradients of the sums, in z (and u); g: the output's gradient
template <bool GATED> __device__ __forceinline__ void finish_backward(const EpiParams& e, const Columns<GATED>& c, uint64_t base, int m, float (&z)[4],
                                                                      float (&u)[4], const float (&g)[4]) {
    float f[4] = {1.0f, 1.0f, 1.0f, 1.0f};
    if (e.drop.threshold) drop_factors<4>((uint64_t)m * (uint64_t)e.N + (uint64_t)c.n, base, e.drop.threshold, e.drop.keep_scale, f);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const bool on = m < e.M && j < c.cnt && f[j] != 0.0f;        // a dropped element's sums do not matter
        float value, slope;
        act_both(fmaf(z[j], e.scale, c.b[j]), e.act, value, slope);
        const float d = g[j] * f[j];
        z[j] = on ? (GATED ? d * fmaf(u[j], e.scale, c.bu[j]) * slope : d * slope) : 0.0f;
        if (GATED) u[j] = on ? d * value : 0.0f;
    }
}
// and their store along the columns, zeros up to `wide`
__device__ __forceinline__ void store_gradient(const EpiParams& e, int m, int n, int half, const float (&d)[4]) {
    if (!e.P || m >= e.M || n >= e.wide) return;                     // wide and n are multiples of 4
    typedef uint16_t u16x4 __attribute__((ext_vector_type(4)));
    u16x4 w[3];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        bf16_t p[3];
        bf16_pieces(d[j], e.pieces, p);
#pragma unroll
        for (int q = 0; q < 3; ++q) w[q][j] = __builtin_bit_cast(uint16_t, p[q]);
    }
    bf16_t* at = e.P + m * e.ldp + half * e.wide + n;
#pragma unroll
    for (int q = 0; q < 3; ++q)
        if (q < e.pieces) *(u16x4*)(at + q * e.p_piece) = w[q];
}

// which tile a workgroup takes: consecutive workgroups go to the eight dies in turn, so that a die gets a contiguous run of tiles, and
// a run goes down eight tiles of m before it moves on in n: both operands of a run are shared in the die's L2
__device__ __forceinline__ void tile_of(int gx, int gy, int id, int& tm, int& tn) {
    const int total = gx * gy, per = total / 8, rem = total % 8, die = id % 8, local = id / 8;
    const int t = die * per + (die < rem ? die : rem) + local;
    const int wide = 8 * gy, group = t / wide, first = group * 8, in = t % wide;
    const int rows = gx - first < 8 ? gx - first : 8;
    tm = first + in % rows;
    tn = in / rows;
}

__device__ const uint32_t lba_zero_piece[4] = {0, 0, 0, 0};

enum { EPI_FORWARD = 0, EPI_BACKWARD = 1 };

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
#pragma unroll
        for (int i = 0; i < 4; ++i) {                    // the code in the high byte of a half: its sign stays, its magnitude moves down
            const uint32_t x = __builtin_amdgcn_perm(0, i < 2 ? w0 : w1, i % 2 ? 0x030c020cu : 0x010c000cu);
            v[i] = (int32_t)((x & 0x80008000u) | ((x >> shift) & keep));
        }
    }
    return v;
}
template <int ELEM> __device__ __forceinline__ f32x4 product_16x16x32(i32x4 b, i32x4 a, f32x4 c) {
    if constexpr (ELEM == ELEM_F16) return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8_t, b), __builtin_bit_cast(f16x8_t, a), c, 0, 0, 0);
    else return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, b), __builtin_bit_cast(bf16x8_t, a), c, 0, 0, 0);
}

// WM x WN waves of FM x FN fragments of 16 x 16
template <int ELEM, int WM, int WN, int FM, int FN, bool GATED, int EPI>
__global__ __launch_bounds__(WM * WN * 64) void dense_kernel(GemmParams p) {
    constexpr int THREADS = WM * WN * 64, BM = WM * FM * 16, BN = WN * FN * 16;
    constexpr int LA = BM * 8 / THREADS, LB = BN * 8 / THREADS;          // pieces a lane stages for a step
    static_assert(BM * 8 % THREADS == 0 && BN * 8 % THREADS == 0 && (!GATED || FN % 2 == 0), "tile");
    __shared__ __attribute__((aligned(16))) uint8_t lds[2][(BM + BN) * 128];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid / 64);
    const int wm = wave / WN, wn = wave % WN;
    int tm, tn;
    tile_of(p.gx, p.gy, blockIdx.x, tm, tn);
    const int m0 = tm * BM, n0 = tn * (GATED ? BN / 2 : BN);

    // staging: lane's rows and its piece of each
    const int piece = (tid & 7) ^ ((tid >> 4) & 7);
    const uint8_t* src[LA + LB];
#pragma unroll
    for (int i = 0; i < LA; ++i) {
        int r = m0 + tid / 8 + i * (THREADS / 8);
        r = r < p.rows_a ? r : p.rows_a - 1;
        src[i] = p.A + r * p.lda + piece * 16;
    }
#pragma unroll
    for (int i = 0; i < LB; ++i) {
        const int t = tid / 8 + i * (THREADS / 8);
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
    const int steps_row = p.steps / p.pieces;
    auto stage = [&](int step, int buf) {
        const int q = p.pieces > 1 ? step / steps_row : 0, s = step - q * steps_row;
        const int64_t off = (int64_t)s * 128, off_a = off + q * p.a_piece;
        auto to_lds = [&](int i, const uint8_t* g) {
            uint8_t* l = &lds[buf][((i < LA ? i : i - LA) * THREADS + wave * 64) * 16 + (i < LA ? 0 : BM * 128)];
            __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) uint32_t*)g,
                                             (__attribute__((address_space(3))) uint32_t*)l, 16, 0, 0);
        };
        if (s * 8 + 8 <= p.chunks) {
#pragma unroll
            for (int i = 0; i < LA + LB; ++i) to_lds(i, src[i] + (i < LA ? off_a : off));
        } else {                                         // the rows end inside this step
            const bool in = s * 8 + piece < p.chunks;
#pragma unroll
            for (int i = 0; i < LA + LB; ++i) to_lds(i, in ? src[i] + (i < LA ? off_a : off) : (const uint8_t*)lba_zero_piece);
        }
    };

    f32x4 acc[FM][FN];
#pragma unroll
    for (int i = 0; i < FM; ++i)
#pragma unroll
        for (int j = 0; j < FN; ++j) acc[i][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};

    const int place = ((lane / 16) ^ ((lane & 15) >> 1)) * 16 + (lane & 15) * 128;
    const int first = p.slices > 1 ? blockIdx.y * p.per_slice : 0;
    const int last = p.slices > 1 ? (first + p.per_slice < p.steps ? first + p.per_slice : p.steps) : p.steps;
    if (first < last) stage(first, 0);
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    for (int step = first; step < last; ++step) {
        const int buf = (step - first) & 1;
        if (step + 1 < last) stage(step + 1, buf ^ 1);
        const uint8_t* la = &lds[buf][wm * FM * 2048 + place];
        const uint8_t* lb = &lds[buf][BM * 128 + wn * FN * 2048 + place];
        // the second piece of a row is 64 bytes on, modulo the row
        const int flip = (place & 64) ? -64 : 64;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            i32x4 rb[FN], ra[FM];
#pragma unroll
            for (int j = 0; j < FN; ++j) rb[j] = *(const i32x4*)(lb + j * 2048 + h * flip);
#pragma unroll
            for (int i = 0; i < FM; ++i) ra[i] = *(const i32x4*)(la + i * 2048 + h * flip);
            if constexpr (ELEM == ELEM_BF16) {
#pragma unroll
                for (int i = 0; i < FM; ++i)
#pragma unroll
                    for (int j = 0; j < FN; ++j) acc[i][j] = product_16x16x32<ELEM>(rb[j], ra[i], acc[i][j]);
            } else {
#pragma unroll
                for (int s = 0; s < 2; ++s) {
                    i32x4 fb[FN];
#pragma unroll
                    for (int j = 0; j < FN; ++j) fb[j] = eight_codes<ELEM>((uint32_t)rb[j][2 * s], (uint32_t)rb[j][2 * s + 1], p.shift_b, p.keep_b);
#pragma unroll
                    for (int i = 0; i < FM; ++i) {
                        const i32x4 fa = eight_codes<ELEM>((uint32_t)ra[i][2 * s], (uint32_t)ra[i][2 * s + 1], p.shift_a, p.keep_a);
#pragma unroll
                        for (int j = 0; j < FN; ++j) acc[i][j] = product_16x16x32<ELEM>(fb[j], fa, acc[i][j]);
                    }
                }
            }
        }
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __syncthreads();
    }

    if (p.split) {                                       // one slice of the sum: raw, for the launch that adds the slices
        const int mr = m0 + wm * FM * 16 + (lane & 15), nr = n0 + (GATED ? wn * FN * 8 : wn * FN * 16) + (lane / 16) * 4;
        float* out = p.split + (int64_t)blockIdx.y * p.e.M * p.rows_b;
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
    // The sums go through LDS, at most 64 rows of a wave at a time, so that neighbouring lanes have neighbouring columns: a wave works on
    // its own part, without barriers.  Place of the four columns c of row r: (c / 4) ^ (r % CH), which spreads a column over the banks.
    constexpr int EH = FM > 4 ? 4 : FM, CH = FN * 4, LPR = GATED ? CH / 2 : CH;      // rows of fragments, fours of a row, lanes of a row
    constexpr int RPP = 64 / LPR, PASSES = EH * 16 / RPP, PB = PASSES < 4 ? PASSES : 4;      // rows of a pass, passes, passes of a batch
    static_assert((PASSES == PB || PASSES % (2 * PB) == 0) && sizeof(lds) >= (size_t)WM * WN * EH * 16 * CH * 16, "epilogue");
    float* mine = (float*)&lds[0][0] + wave * (EH * 16 * CH * 4);
    const uint64_t base = p.e.drop.threshold ? drop_base(p.e.drop) : 0;
    const int quad = lane % LPR, row_in = lane / LPR;
    const int cz = GATED ? quad / 4 * 8 + quad % 4 : quad;                           // its place in the row of sums
    const int ncol = n0 + wn * (GATED ? FN * 8 : FN * 16) + quad * 4;
    const Columns<GATED> cols = columns_of<GATED>(p.e, ncol);
    const void* extra = EPI == EPI_FORWARD ? p.e.R : p.e.G;
    const int extra_type = EPI == EPI_FORWARD ? p.e.r_type : p.e.g_type;
    float sz[4] = {0.0f, 0.0f, 0.0f, 0.0f}, su[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int h = 0; h < FM / EH; ++h) {
        const int mh = m0 + (wm * FM + h * EH) * 16;
        float x[2][PB][4];            // a batch's residuals or gradients are on their way while the one before is worked on
        if (extra) {
#pragma unroll
            for (int q = 0; q < PB; ++q) load_extra(p.e, extra, extra_type, mh + q * RPP + row_in, ncol, x[0][q]);
        }
#pragma unroll
        for (int i = 0; i < EH; ++i)
#pragma unroll
            for (int j = 0; j < FN; ++j) {
                const int r = i * 16 + (lane & 15), c = j * 4 + lane / 16;
                *(f32x4*)(mine + (r * CH + (c ^ (r % CH))) * 4) = acc[h * EH + i][j];
            }
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
        __builtin_amdgcn_wave_barrier();
#pragma unroll 1
        for (int g = 0; g < PASSES; g += 2 * PB) {
#pragma unroll
            for (int part = 0; part < 2; ++part) {
                if (PASSES > PB || part == 0) {
                    const int g0 = g + part * PB;
                    if (extra && g0 + PB < PASSES) {
#pragma unroll
                        for (int q = 0; q < PB; ++q) load_extra(p.e, extra, extra_type, mh + (g0 + PB + q) * RPP + row_in, ncol, x[part ^ 1][q]);
                    }
#pragma unroll
                    for (int q = 0; q < PB; ++q) {
                        const int r = (g0 + q) * RPP + row_in, m = mh + r;
                        float* at = mine + (r * CH + (cz ^ (r % CH))) * 4;
                        float* at2 = mine + (r * CH + ((cz + 4) ^ (r % CH))) * 4;
                        float z[4], u[4] = {0.0f, 0.0f, 0.0f, 0.0f};
                        const f32x4 vz = *(const f32x4*)at;
#pragma unroll
                        for (int k = 0; k < 4; ++k) z[k] = vz[k];
                        if (GATED) {
                            const f32x4 vu = *(const f32x4*)at2;
#pragma unroll
                            for (int k = 0; k < 4; ++k) u[k] = vu[k];
                        }
                        if constexpr (EPI == EPI_FORWARD) {
                            finish_forward<GATED>(p.e, cols, base, m, z, u, x[part][q]);
                        } else {
                            finish_backward<GATED>(p.e, cols, base, m, z, u, x[part][q]);
                            store_gradient(p.e, m, ncol, 0, z);
                            if (GATED) store_gradient(p.e, m, ncol, 1, u);
                            *(f32x4*)at = f32x4{z[0], z[1], z[2], z[3]};
                            if (GATED) *(f32x4*)at2 = f32x4{u[0], u[1], u[2], u[3]};
#pragma unroll
                            for (int k = 0; k < 4; ++k) { sz[k] += z[k]; su[k] += u[k]; }
                        }
                    }
                }
            }
        }
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
        __builtin_amdgcn_wave_barrier();
        if constexpr (EPI == EPI_BACKWARD) {
            if (p.e.PT) {                                // the transposed copy: eight rows of one column a lane
                constexpr int LM = EH * 2, NPP = 64 / LM;                            // lanes along m, columns of a pass
                const int r0 = (lane % LM) * 8, m = mh + r0;
#pragma unroll 1
                for (int c0 = 0; c0 < CH * 4; c0 += NPP) {
                    const int c = c0 + lane / LM;
                    const int n = n0 + wn * (GATED ? FN * 8 : FN * 16) + (GATED ? c / 32 * 16 + c % 16 : c);
                    const int half = GATED ? c / 16 % 2 : 0;
                    typedef uint16_t u16x8 __attribute__((ext_vector_type(8)));
                    u16x8 w[3];
#pragma unroll
                    for (int k = 0; k < 8; ++k) {
                        const int r = r0 + k;
                        bf16_t b[3];
                        bf16_pieces(mine[(r * CH + ((c / 4) ^ (r % CH))) * 4 + c % 4], p.e.pieces, b);
#pragma unroll
                        for (int q = 0; q < 3; ++q) w[q][k] = __builtin_bit_cast(uint16_t, b[q]);
                    }
                    if (n < p.e.N && m < p.e.ldt) {      // ldt and m are multiples of 8: zeros beyond M are part of the copy
                        bf16_t* at = p.e.PT + ((int64_t)half * p.e.N + n) * p.e.ldt + m;
#pragma unroll
                        for (int q = 0; q < 3; ++q)
                            if (q < p.e.pieces) *(u16x8*)(at + q * p.e.pt_piece) = w[q];
                    }
                }
                __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
                __builtin_amdgcn_wave_barrier();
            }
        }
    }
    if constexpr (EPI == EPI_BACKWARD) {
        if (p.e.part) {                                  // column sums of the wave's rows: over the lanes that share a column
#pragma unroll
            for (int k = 0; k < 4; ++k) {
#pragma unroll
                for (int d = LPR; d < 64; d *= 2) {
                    sz[k] += __shfl_xor(sz[k], d);
                    if (GATED) su[k] += __shfl_xor(su[k], d);
                }
            }
            if (row_in == 0 && ncol < p.e.N) {
                float* out = p.e.part + (int64_t)(tm * WM + wm) * (GATED ? 2 * p.e.N : p.e.N);
                store_some<4>(out + ncol, p.e.N - ncol, sz, p.e.fmt);
                if (GATED) store_some<4>(out + p.e.N + ncol, p.e.N - ncol, su, p.e.fmt);
            }
        }
    }
}

// tiles: rows of outputs, columns of B and waves over m
enum { TILE_256 = 0, TILE_128 = 1, TILE_64 = 2 };
struct TileShape { int bm, bn, wm; };
inline TileShape tile_shape(int tile) { return tile == TILE_256 ? TileShape{256, 256, 2} : tile == TILE_128 ? TileShape{128, 128, 2} : TileShape{64, 64, 2}; }

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

// A format as the kernels read it: how its codes become 16-bit operands, and the factor that is left (value = operand * factor).
struct ElemFmt { int elem, shift; uint32_t keep; float factor; };
inline ElemFmt make_elem(const lba_infmt& f, int elem) {
    const int bc = (1 << (f.exp_bits - 1)) - 1;
    ElemFmt e = {elem, f.man_bits - 2, (0x7Fu << (10 - f.man_bits)) * 0x10001u, 0.0f};
    e.factor = __builtin_ldexpf(1.0f, elem == ELEM_F16 ? 15 - f.bias : bc - f.bias);
    return e;
}
// one kind for both operands of a product
inline int elem_of(const lba_infmt& a, const lba_infmt& b) {
    if (a.exp_bits == 4 && b.exp_bits == 4) return ELEM_E4M3;
    return a.exp_bits <= 4 && b.exp_bits <= 4 ? ELEM_F16 : ELEM_BF16;
}

// few rows (at most kTokenRows): a pass over B (lba_dense_token.hip)
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

// launches a product whose parameters are complete but for the grid
void launch_dense_e4m3(GemmParams& p, int tile, bool gated, int epi, hipStream_t st);
void launch_dense_f16(GemmParams& p, int tile, bool gated, int epi, hipStream_t st);
void launch_dense_bf16(GemmParams& p, int tile, bool gated, int epi, hipStream_t st);

template <int ELEM> void launch_dense(GemmParams& p, int tile, bool gated, int epi, hipStream_t st) {
    const TileShape s = tile_shape(tile);
    p.gx = (p.e.M + s.bm - 1) / s.bm;
    p.gy = gated ? (p.half + s.bn / 2 - 1) / (s.bn / 2) : (p.rows_b + s.bn - 1) / s.bn;
    const dim3 grid((unsigned)(p.gx * p.gy), (unsigned)(p.slices > 1 ? p.slices : 1));
#define LBA_DENSE(TILE, WM, WN, FM, FN, GATED, EPI) \
    if (tile == TILE && gated == GATED && epi == EPI) { \
        hipLaunchKernelGGL((dense_kernel<ELEM, WM, WN, FM, FN, GATED, EPI>), grid, dim3(WM * WN * 64), 0, st, p); \
        return; \
    }
#define LBA_DENSE_TILES(GATED, EPI) \
    LBA_DENSE(TILE_256, 2, 4, 8, 4, GATED, EPI) LBA_DENSE(TILE_128, 2, 2, 4, 4, GATED, EPI) LBA_DENSE(TILE_64, 2, 2, 2, 2, GATED, EPI)
    LBA_DENSE_TILES(false, EPI_FORWARD)
    LBA_DENSE_TILES(true, EPI_FORWARD)
    LBA_DENSE_TILES(false, EPI_BACKWARD)
    LBA_DENSE_TILES(true, EPI_BACKWARD)
#undef LBA_DENSE_TILES
#undef LBA_DENSE
}

}  // namespace lba
#endif

// lba_dense_token.hip -- the dense product of a few rows: single tokens, short batches of them.
//
// With M rows a product does 2 M operations for each code of B, so up to M of a few hundred it is a pass over B.  A workgroup owns
// sixteen columns (gated: of both halves) and its eight waves take steps of 128 codes of k in turn: lane l reads 32 consecutive codes
// of row l % 16 straight into the registers of a matrix-core fragment, no LDS in between, and the waves' sums meet in LDS at the end,
// always in the same order.  Codes become bfloat16 or FP16 numbers in registers (lba_dense.h says why).  Rows may start anywhere; only a
// last step that the row does not fill is read code by code.
// Bound by the pass over B: 1 x 4096 x 4096 in 6.2 us, 2.7 TB/s, 6 x (2 x 4096) x 2048 gated 5.7 us; a launch of one small workgroup takes 3.
// With codes of five exponent bits by their conversion, which is arithmetic: 12 us where E4M3 takes 5.2 and M4E3 5.7 with B in the last-level
// cache.  lba_dense.h has it beside the tile, from 1 to 64 rows.
#include "lba_dense.h"

namespace lba {

typedef i32x4 i32x4_any __attribute__((aligned(1)));

struct Codes32 { i32x4 a, b; };

// codes k .. k + 31 of a row that ends at K; what is past the end reads as code 0
__device__ __forceinline__ Codes32 load_codes(const uint8_t* row, int k, int K) {
    Codes32 c;
    if (k + 32 <= K) {
        c.a = *(const i32x4_any*)(row + k);
        c.b = *(const i32x4_any*)(row + k + 16);
        return c;
    }
    uint32_t w[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        w[i] = 0;
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (k + 4 * i + j < K) w[i] |= (uint32_t)row[k + 4 * i + j] << (8 * j);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) { c.a[i] = (int32_t)w[i]; c.b[i] = (int32_t)w[4 + i]; }
    return c;
}

template <int ELEM> __device__ __forceinline__ i32x4 eighth(const Codes32& c, int q, const ElemFmt& f, const CodeBits& bits) {
    const i32x4& h = q < 2 ? c.a : c.b;
    const uint32_t w0 = (uint32_t)h[(q & 1) * 2], w1 = (uint32_t)h[(q & 1) * 2 + 1];
    if constexpr (ELEM == ELEM_BF16) {                   // five exponent bits: any format by arithmetic
        uint32_t w[4];
        code_bf16(w0, bits, w[0], w[1]);
        code_bf16(w1, bits, w[2], w[3]);
        return i32x4{(int32_t)w[0], (int32_t)w[1], (int32_t)w[2], (int32_t)w[3]};
    } else {
        return eight_codes<ELEM>(w0, w1, f.shift, f.keep);
    }
}

template <int ELEM, bool GATED, int MF>
__global__ __launch_bounds__(512) void dense_token_kernel(TokenParams p) {
    constexpr int W = 8, H = GATED ? 2 : 1;
    __shared__ f32x4 sums[W][MF * H][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x / 64;
    const int n0 = blockIdx.x * 16;
    const int lim = GATED ? p.half : p.rows_b;
    const int nb = n0 + (lane & 15) < lim ? n0 + (lane & 15) : lim - 1;
    const uint8_t* b0 = p.B + (int64_t)nb * p.K;
    const uint8_t* b1 = b0 + (GATED ? (int64_t)p.half * p.K : 0);
    const uint8_t* a[MF];
#pragma unroll
    for (int f = 0; f < MF; ++f) {
        const int m = f * 16 + (lane & 15);
        a[f] = p.A + (int64_t)(m < p.M ? m : p.M - 1) * p.K;
    }
    f32x4 acc[MF][H];
#pragma unroll
    for (int f = 0; f < MF; ++f)
#pragma unroll
        for (int h = 0; h < H; ++h) acc[f][h] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    for (int k = wave * 128; k < p.K; k += W * 128) {
        const int kl = k + (lane / 16) * 32;
        Codes32 cb[H], ca[MF];
        cb[0] = load_codes(b0, kl, p.K);
        if (GATED) cb[H - 1] = load_codes(b1, kl, p.K);
#pragma unroll
        for (int f = 0; f < MF; ++f) ca[f] = load_codes(a[f], kl, p.K);
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            i32x4 vb[H];
#pragma unroll
            for (int h = 0; h < H; ++h) vb[h] = eighth<ELEM>(cb[h], q, p.fb, p.cb);
#pragma unroll
            for (int f = 0; f < MF; ++f) {
                const i32x4 va = eighth<ELEM>(ca[f], q, p.fa, p.ca);
#pragma unroll
                for (int h = 0; h < H; ++h) acc[f][h] = product_16x16x32<ELEM>(vb[h], va, acc[f][h]);
            }
        }
    }
#pragma unroll
    for (int f = 0; f < MF; ++f)
#pragma unroll
        for (int h = 0; h < H; ++h) sums[wave][f * H + h][lane] = acc[f][h];
    __syncthreads();
    if (wave >= MF) return;
    const int m = wave * 16 + (lane & 15);
    const Columns<GATED, 4> cols = columns_of<GATED, 4>(p.e, n0 + (lane / 16) * 4);
    float r[4];
    load_extra<4>(p.e, m, cols.n, r);
    f32x4 s[H];
#pragma unroll
    for (int h = 0; h < H; ++h) {
        s[h] = sums[0][wave * H + h][lane];
#pragma unroll
        for (int w = 1; w < W; ++w) s[h] += sums[w][wave * H + h][lane];
    }
    float z[4], u[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) { z[j] = s[0][j]; u[j] = s[H - 1][j]; }
    const uint64_t base = p.e.drop.on ? drop_base(p.e.drop) : 0;
    with_act(p.e.act, [&](auto act) { finish_forward<GATED, false, decltype(act)::value, 4>(p.e, cols, base, m, At{(int64_t)m * p.e.N + cols.n, 0}, z, u, r); });
}

void launch_dense_token(const TokenParams& p, int elem, bool gated, hipStream_t st) {
    const int mf = (p.M + 15) / 16;
    const dim3 grid((unsigned)(((gated ? p.half : p.rows_b) + 15) / 16));
#define LBA_TOKEN(EL, GA, MF) \
    if (elem == EL && gated == GA && mf == MF) { hipLaunchKernelGGL((dense_token_kernel<EL, GA, MF>), grid, dim3(512), 0, st, p); return; }
#define LBA_TOKEN_ROWS(EL, GA) LBA_TOKEN(EL, GA, 1) LBA_TOKEN(EL, GA, 2) LBA_TOKEN(EL, GA, 3) LBA_TOKEN(EL, GA, 4)
    LBA_TOKEN_ROWS(ELEM_E4M3, false) LBA_TOKEN_ROWS(ELEM_E4M3, true) LBA_TOKEN_ROWS(ELEM_F16, false)
    LBA_TOKEN_ROWS(ELEM_F16, true) LBA_TOKEN_ROWS(ELEM_BF16, false) LBA_TOKEN_ROWS(ELEM_BF16, true)
#undef LBA_TOKEN_ROWS
#undef LBA_TOKEN
}

}  // namespace lba

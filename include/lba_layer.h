/* lba_layer.h -- C ABI of the operators around the products of a transformer layer: layer norm, dropout with bias, activation
 * and residual, the dense product of 8-bit codes with wide accumulators, and the gated feed-forward product, each with its
 * backward pass.
 *
 * The simulated products of lba.h take 8-bit codes and return float32 sums; what stands between two of them in a layer is here,
 * with codes as one of the output types, so that a result is the next product's operand.  lba_dense is the product that the
 * simulated one is compared with and trained from: the same codes, exact products, float32 accumulation on the matrix cores.
 *
 * As in lba.h: all pointers are DEVICE pointers owned by the caller, matrices are row-major and contiguous, calls enqueue work on
 * `hip_stream` and return without synchronising, the library keeps no state between calls and allocates no device memory, nothing
 * is enqueued on an error, and no alignment is required of any argument but a workspace (256 bytes, else LBA_ERR_ALIGN).
 * No call uses atomic additions: the same inputs give the same bits on every run.  Inputs and outputs must not overlap, except
 * that an output may be the same array as an input of the same type where a call says so. */
#ifndef LBA_LAYER_H_
#define LBA_LAYER_H_

#include "lba.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Element types.  LBA_CODE8: 8-bit codes of an lba_infmt (lba.h), whose bias carries the tensor's power-of-two scale: the codes of
 * {4, 3, 7 + t} are the E4M3 codes of x * 2^t.  Written codes are rounded to nearest, ties to even, and saturate at the largest
 * value of the format (exp_bits 4: +-448 of the canonical bias, the codes 0x7f and 0xff are not written for numbers); a NaN is
 * written as 0x7f or 0xff. */
enum { LBA_F32 = 0, LBA_BF16 = 1, LBA_CODE8 = 2 };

/* Activations: none, max(z, 0), z * Phi(z) with the normal distribution function Phi, z / (1 + exp(-z)). */
enum { LBA_ACT_NONE = 0, LBA_ACT_RELU = 1, LBA_ACT_GELU = 2, LBA_ACT_SILU = 3 };

/* Dropout.  Element i (its index in the whole output) is dropped iff u_i < T with T = floor(65536 p + 1/2), and what stays is
 * multiplied by 65536 / (65536 - T): the rate applied is p rounded to 16 bits, and its complement is exact.
 *   u_i = bits 16 (i % 4) .. + 15 of mix(base + floor(i / 4) * g),   g = 0x9E3779B97F4A7C15
 *   base = mix(mix(2 seed + 1) ^ (2 (stream + step) + 1) * g),   mix = the splitmix64 finaliser, everything modulo 2^64
 * `step` points to one device word (NULL: 0) that is read when the kernel runs, so that a captured graph draws a new mask at every
 * replay.  Nothing of the mask is stored: the backward pass makes it again.  p must be in [0, 1] (else LBA_ERR_FORMAT); p = 0
 * (T = 0) drops nothing, p = 1 everything.  A dropped element's value does not matter, infinities and NaN included. */
typedef struct {
    double p;
    uint64_t seed, stream;
    const uint64_t* step;
} lba_drop;

/* Layer norm over rows of length N (M rows):  y = (x - mean) * rstd * gamma + beta, rstd = (var + eps)^-1/2, var the mean of
 * (x - mean)^2, all in float32; with codes for Y and N <= 16384 in 64 bits, so that the codes are the nearest to the exact result.
 * X [M, N] of x_type (LBA_F32 or LBA_BF16), gamma and beta [N] float32 (NULL: ones, zeros), Y [M, N] of y_type (y_fmt is read for
 * LBA_CODE8 only), mean and rstd [M] float32 (either may be NULL: not stored).  Y may be X where the types are equal.
 * M <= 2^31 - 1, N <= 2^21 (else LBA_ERR_SHAPE).  N == 0: mean and rstd are NaN. */
int lba_layernorm(const void* X, int32_t x_type, const float* gamma, const float* beta, float eps,
                  void* Y, int32_t y_type, lba_infmt y_fmt, float* mean, float* rstd,
                  int64_t M, int64_t N, void* hip_stream);

/* Its gradients.  With n = (x - mean) * rstd, h = G * gamma, and means over a row,
 *   dX = rstd * (h - mean(h) - n * mean(h * n)),   dgamma = sum over rows of G * n,   dbeta = sum over rows of G.
 * G [M, N] of g_type, X as in the forward call, mean and rstd as it stored them; dX [M, N] of x_type, dgamma and dbeta [N] float32;
 * any of the three may be NULL but not all (unless M or N is 0).  dX may be G or X where the types are equal.  M == 0 stores zeros to
 * dgamma and dbeta.
 * workspace: lba_layernorm_bwd_workspace_bytes(M, N) bytes (needed for dgamma or dbeta only). */
int lba_layernorm_bwd(const void* G, int32_t g_type, const void* X, int32_t x_type, const float* gamma,
                      const float* mean, const float* rstd, void* dX, float* dgamma, float* dbeta,
                      int64_t M, int64_t N, void* workspace, size_t workspace_bytes, void* hip_stream);
size_t lba_layernorm_bwd_workspace_bytes(int64_t M, int64_t N);

/* Y = residual + keep * act(scale * X + bias) / (1 - p), what follows a simulated product (scale = 2^-T undoes its operands'
 * scales).  X [M, N] of x_type, bias [N] float32 or NULL, residual [M, N] of r_type or NULL, Y [M, N] of y_type.  Y may be X or residual
 * where the types are equal.  M <= 2^31 - 1, N <= 2^21. */
int lba_dropout(const void* X, int32_t x_type, float scale, const float* bias, int32_t act, lba_drop drop,
                const void* residual, int32_t r_type, void* Y, int32_t y_type, lba_infmt y_fmt,
                int64_t M, int64_t N, void* hip_stream);

/* Its gradients:  dZ = G * keep / (1 - p) * act'(scale * X + bias),  dX = scale * dZ,  dbias = sum over rows of dZ (either may be
 * NULL but not both, unless M or N is 0; the residual's gradient is G itself).  M == 0 stores zeros to dbias.  act' of LBA_ACT_RELU is
 * 0 at 0.  X and bias are read only where act is not LBA_ACT_NONE.  dX is of x_type and may be G or X where the types are equal.
 * workspace: lba_dropout_bwd_workspace_bytes(M, N) bytes (needed for dbias only). */
int lba_dropout_bwd(const void* G, int32_t g_type, const void* X, int32_t x_type, float scale, const float* bias,
                    int32_t act, lba_drop drop, void* dX, float* dbias, int64_t M, int64_t N,
                    void* workspace, size_t workspace_bytes, void* hip_stream);
size_t lba_dropout_bwd_workspace_bytes(int64_t M, int64_t N);

/* The product of 8-bit codes with float32 accumulation, and what follows it, in one call:
 *   gated == 0:  Y = residual + keep * act(S + bias) / (1 - p),                     S = value(A) . value(B)^T,   B [N, K]
 *   gated != 0:  Y = residual + keep * act(S_g + b_g) * (S_u + b_u) / (1 - p),      B [2 N, K], bias [2 N]: the gate's N rows first
 * A [M, K] codes of fmt_a, B codes of fmt_b (the biases of the formats are the operands' scales: S is in real units), bias float32 or NULL,
 * residual [M, N] of r_type or NULL, Y [M, N] of y_type.  Products are exact and sums are float32.  The NaN codes of E4M3 are outside the
 * contract, as in lba.h: the outputs they reach are unspecified.  K == 0: S = 0.
 * Limits (else LBA_ERR_SHAPE): M <= 2^30, N <= 2^20, K <= 2^30, and with more than 64 rows fewer than 2^23 tiles of 256 x 256:
 * ceil(M / 256) * ceil(rows of B / 256) < 2^23; (else LBA_ERR_FORMAT): the formats' limits of lba.h.
 * workspace: lba_dense_workspace_bytes(...) bytes, NULL where that is 0; `aligned`: A and B are 16-byte aligned.  Operands of at most 4
 * exponent bits whose rows are multiples of 16 bytes are used where they are, and those of at most 64 rows of A in any case; others are copied
 * there, and codes of 5 exponent bits as bfloat16, which holds them: then (M + 64) (K + 64) and (rows of B + 64) (K + 64) must not exceed
 * 2^32 (else LBA_ERR_SHAPE). */
int lba_dense(const uint8_t* A, const uint8_t* B, int64_t M, int64_t N, int64_t K, lba_infmt fmt_a, lba_infmt fmt_b, int32_t gated,
              const float* bias, int32_t act, lba_drop drop, const void* residual, int32_t r_type,
              void* Y, int32_t y_type, lba_infmt y_fmt, void* workspace, size_t workspace_bytes, void* hip_stream);
size_t lba_dense_workspace_bytes(int64_t M, int64_t N, int64_t K, lba_infmt fmt_a, lba_infmt fmt_b, int32_t gated, int32_t aligned);

/* Its gradients.  Nothing of the forward call is kept: where act or gated needs S, it is computed again.  With G = dL/dY [M, N] of
 * g_type and D the gradient of the sums ([M, N], gated [M, 2 N]: the gate's columns first),
 *   dA = D . value(B) [M, K],   dB = D^T . value(A) [N or 2 N, K],   dbias = sum over rows of D (float32); the residual's gradient is G.
 * dA and dB are of g_type and gradients of the operands' real values; any of the three may be NULL but not all (unless M, N or K is 0).
 * Sums over nothing store zeros.  Float32: D is split exactly into three bfloat16 pieces and the products are exact, sums float32 (a
 * value of D under 2^-100 may lose pieces to the flush of subnormal numbers, an infinite one gives NaN).  Bfloat16: D is rounded to
 * bfloat16 before the two products, as dA and dB are after them; dbias sums D before that.
 * Limits: M, N, K and formats as in lba_dense, (M + 64) (K + 64), (rows of B + 64) (K + 64) <= 2^32 for any operands, and
 * ceil(M / 128) * ceil(rows of B / 128) < 3 * 2^22.
 * workspace: lba_dense_bwd_workspace_bytes(...) bytes. */
int lba_dense_bwd(const void* G, int32_t g_type, const uint8_t* A, const uint8_t* B, int64_t M, int64_t N, int64_t K,
                  lba_infmt fmt_a, lba_infmt fmt_b, int32_t gated, const float* bias, int32_t act, lba_drop drop,
                  void* dA, void* dB, float* dbias, void* workspace, size_t workspace_bytes, void* hip_stream);
size_t lba_dense_bwd_workspace_bytes(int64_t M, int64_t N, int64_t K, lba_infmt fmt_a, lba_infmt fmt_b, int32_t gated, int32_t act,
                                     int32_t g_type, int32_t aligned);

#ifdef __cplusplus
}
#endif
#endif /* LBA_LAYER_H_ */

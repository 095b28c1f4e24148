/* lba_attention.h -- C ABI of what stands between the query, key and value product of a transformer layer and its output product: rotary
 * positions, attention over packed sequences (each with its backward pass), a cache of keys and values that holds 4 bits an element, and
 * attention of new tokens over it.
 *
 * The products before and after are those of lba.h and lba_layer.h: lba_dense writes the queries, keys and values side by side, the calls here
 * read them where they are, and attention can write the codes that the output product reads.
 *
 * As in lba_layer.h: all pointers are DEVICE pointers owned by the caller, calls enqueue work on `hip_stream` and return without
 * synchronising, the library keeps no state between calls and allocates no device memory, nothing is enqueued on an error, no call uses
 * atomic additions (the same inputs give the same bits on every run), and no alignment is required of any argument but a workspace (256
 * bytes, else LBA_ERR_ALIGN) beyond that of its elements.  Inputs and outputs must not overlap, except where a call says so.
 *
 * Tensors of heads have rows of one token each: element d of head h of row t is at t * row + h * head + d, counted in elements.  Strides
 * must not be negative (else LBA_ERR_SHAPE), and no two elements of an output may share a place. */
#ifndef LBA_ATTENTION_H_
#define LBA_ATTENTION_H_

#include "lba_layer.h"

#ifdef __cplusplus
extern "C" {
#endif

/* May be added to the type of the inputs of lba_attention, lba_attention_bwd and lba_cache_attention, where it is said what it asks for. */
#define LBA_FINE 0x100

typedef struct {
    int64_t row, head;
} lba_strides;

/* Rotary positions.  With `pairs` frequencies f_i (radians a position, float64), the first 2 * pairs elements of each of the H heads of a row
 * are taken as pairs, (i, i + pairs) or, interleaved, (2 i, 2 i + 1), and each pair (a, b) of a row with position m becomes
 *   gain * (a cos(m f_i) - b sin(m f_i)),   gain * (b cos(m f_i) + a sin(m f_i)).
 * The other elements are copied.  Angles are products in float64, reduced to a part of a turn there; cosine, sine and the rotation are float32.
 * X and Y [T, H, D] of `type` (LBA_F32 or LBA_BF16); Y may be X with the same strides.  positions: T integers of pos_bits (32 or 64) bits, of
 * either sign.  Limits (else LBA_ERR_SHAPE): T <= 2^31 - 1, H <= 65535, D <= 1024, 2 * pairs <= D. */
int lba_rope(const void* X, lba_strides x_at, int32_t type, const void* positions, int32_t pos_bits, const double* freq, int64_t pairs,
             int32_t interleaved, float gain, void* Y, lba_strides y_at, int64_t T, int64_t H, int64_t D, void* hip_stream);

/* Its gradient: with G = dL/dY, dX is G rotated back, gain * (a cos + b sin), gain * (b cos - a sin), and G where Y is a copy.  dX may be G
 * with the same strides. */
int lba_rope_bwd(const void* G, lba_strides g_at, int32_t type, const void* positions, int32_t pos_bits, const double* freq, int64_t pairs,
                 int32_t interleaved, float gain, void* dX, lba_strides dx_at, int64_t T, int64_t H, int64_t D, void* hip_stream);

/* Packed sequences.  Sequence b has the query rows starts[b] .. starts[b + 1] - 1 of T and the key rows starts_k[b] .. starts_k[b + 1] - 1 of
 * Tk; both lists hold count + 1 integers that never fall, from 0 or more to T (Tk) or less.  starts_k NULL: as starts.  Both NULL: `count`
 * sequences of equal length, T / count and Tk / count (else LBA_ERR_SHAPE).  Lists that break this give unspecified rows, but nothing
 * outside the tensors is read or written.
 * Query head h reads head h / (H / KV) of the keys and values (H a multiple of KV, else LBA_ERR_SHAPE).  Query i of n sees key j of m iff
 * causal == 0 or j <= i + m - n: the last query sees all.  What is hidden does not matter, infinities and NaN included.
 * Rows of no sequence are left as they were, or, clear != 0, stored as zeros (-infinity in lse).
 * Q, K and V of `type` (LBA_F32 or LBA_BF16).  Float32 factors of products are three bfloat16 pieces, which hold them (numbers of 2^-100 or more
 * in size); of the nine products of pieces the six largest are summed, the others are under 2^-24 of the whole.
 * Limits (else LBA_ERR_SHAPE): T, Tk <= 2^31 - 1, count <= 2^20, H <= 65535, 1 <= D <= 128, and (rows / 128 + count) * heads <= 2^23 for the query
 * rows with H and for the key rows with KV. */
typedef struct {
    int64_t T, Tk, count;
    const int32_t *starts, *starts_k;
    int32_t H, KV, D, type, causal, clear;
    float scale;
    lba_strides q, k, v;
} lba_attn;

/* O = softmax over the seen keys of (scale * q . k) times V; a query that sees nothing, or whose scores are all -infinity, has
 * zeros.  Scores, the softmax's maximum and sum and O's sums are float32; with LBA_BF16 and an output of
 * another type than LBA_F32 the weights are rounded to bfloat16 for the product with V, unless LBA_FINE is added to a.type: they are three
 * bfloat16 pieces then, which hold them, as with LBA_F32.
 * O [T, H, D] contiguous of o_type (o_fmt is read for LBA_CODE8 only); lse [T, H] float32 (NULL: not stored): ln of the sum over the seen
 * keys of exp(scale * q . k), -infinity where there are none.
 * workspace: lba_attention_workspace_bytes(a) bytes, which reads no pointer of `a` but whether it is NULL; 0 where there are many rows. */
int lba_attention(lba_attn a, const void* Q, const void* K, const void* V, void* O, int32_t o_type, lba_infmt o_fmt, float* lse, void* workspace,
                  size_t workspace_bytes, void* hip_stream);
size_t lba_attention_workspace_bytes(lba_attn a);

/* Its gradients.  With P the weights, made again from lse, and G = dL/dO,
 *   dV = P^T . G,   S = P * (G . V^T - rowsum(G * O)),   dQ = scale * S . K,   dK = scale * S^T . Q,
 * summed over the query heads of a key head.  Gradients that a seen infinity or NaN reaches are unspecified.  G and O
 * [T, H, D] contiguous, all of a.type, O and lse as the forward call stored them; dQ [T, H, D], dK and dV [Tk, KV, D] of a.type.  With LBA_BF16 P and S are rounded to bfloat16 for the
 * products; sums are float32.  rowsum(G * O) is the sum of P * (G . V^T) where a query's tile of 128 sees up to 512 keys, and, with LBA_FINE added
 * to a.type, of all queries; else it is taken from O as it is stored, whose rounding tells where values have a mean.
 * workspace: lba_attention_bwd_workspace_bytes(a) bytes. */
int lba_attention_bwd(lba_attn a, const void* G, const void* Q, const void* K, const void* V, const void* O, const float* lse, void* dQ,
                      lba_strides dq_at, void* dK, lba_strides dk_at, void* dV, lba_strides dv_at, void* workspace, size_t workspace_bytes,
                      void* hip_stream);
size_t lba_attention_bwd_workspace_bytes(lba_attn a);

/* A cache of keys and values in 4 bits.  Each 32 consecutive elements of a head are held as a power of two, one byte e for 2^(e - 127) (0: for zero), and
 * 4-bit codes, two a byte, the first in the low half: sign, two exponent bits, one mantissa bit, the numbers 0, 0.5, 1, 1.5, 2, 3, 4, 6 and
 * their negatives.  Written blocks have the smallest power for which the largest element is at most 6 of it, within 2^-100 .. 2^125, and
 * elements rounded to nearest, ties to even, saturating; elements under 2^-126 in size count as zero, a block with an infinity or a NaN is
 * written as e = 255, which reads as NaN.
 * k, v: codes [pages, KV, page, D / 2]; k_scale, v_scale: [pages, KV, page, D / 32].  D is 32, 64, 96 or 128 (else LBA_ERR_SHAPE),
 * page 1 .. 2^16, pages <= 2^31 - 1.
 * Sequence b's token at position p is in page table[b * table_row + p / page], line p % page; the table has table_row >= 0 pages for each of
 * `count` sequences and lens[b] tokens are in use.  Positions beyond the table and pages outside 0 .. pages - 1 hold nothing: what is
 * written there is dropped, read as zero, and not seen by a query.
 * Limits (else LBA_ERR_SHAPE): count <= 2^20, table_row <= 2^31 - 1, KV <= 65535. */
typedef struct {
    uint8_t *k, *k_scale, *v, *v_scale;
    int64_t pages, table_row, count;
    const int32_t *table, *lens;
    int32_t page, KV, D;
} lba_cache4;

/* Writes the newest tokens: rows starts[b] .. starts[b + 1] - 1 of K and V ([T, KV, D] of `type`) go to positions
 * lens[b] - (starts[b + 1] - starts[b]) .. lens[b] - 1 of sequence b (lens counts them); those below 0 are dropped.  starts NULL: T / count rows
 * each.  Two rows that go to one place leave a mix of the two there. */
int lba_cache_write(lba_cache4 c, const int32_t* starts, int64_t T, const void* K, lba_strides k_at, const void* V, lba_strides v_at, int32_t type,
                    void* hip_stream);

/* Reads the newest tokens back, in the same arrangement, exactly (numbers under 2^-126 in size as they are or as zero): K and V [T, KV, D] of `type`.
 * Positions below 0 read as zeros.  Rows of no sequence are left as they were, or, clear != 0, stored as zeros. */
int lba_cache_read(lba_cache4 c, const int32_t* starts, int64_t T, void* K, lba_strides k_at, void* V, lba_strides v_at, int32_t type, int32_t clear,
                   void* hip_stream);

/* Attention of each sequence's `fresh` newest tokens over its cache: query i of a sequence (Q [count, fresh, H, D], a token's strides q_at, of `type`)
 * sees positions 0 .. lens[b] - fresh + i, as far as they hold something.  O [count, fresh, H, D] contiguous of o_type; a query that sees nothing has zeros.
 * Scores, maxima and sums are float32; with LBA_BF16 and an output of another type than LBA_F32 the weights are rounded to bfloat16 for the
 * product with the values, else, and with LBA_FINE added to type, they are split into three bfloat16 pieces, which hold them, as queries of LBA_F32 are.
 * Limits (else LBA_ERR_SHAPE): H a multiple of KV, H <= 65535, count * fresh * H < 2^24, table_row * page <= 2^30, and with tiles of 16 rows (the fresh
 * queries of the H / KV heads that share one; 32 where there are more) tiles * KV * count < 2^23.
 * workspace: lba_cache_attention_workspace_bytes(...) bytes, for the longest sequence that the table has room for. */
int lba_cache_attention(lba_cache4 c, const void* Q, lba_strides q_at, int32_t type, int64_t fresh, int64_t H, float scale, void* O, int32_t o_type,
                        lba_infmt o_fmt, void* workspace, size_t workspace_bytes, void* hip_stream);
size_t lba_cache_attention_workspace_bytes(int64_t count, int64_t table_row, int32_t page, int64_t fresh, int64_t H, int32_t KV, int32_t D);

#ifdef __cplusplus
}
#endif
#endif /* LBA_ATTENTION_H_ */

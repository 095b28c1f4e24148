// lba_attn.hip -- attention over packed sequences, forward: one wave to a query row of a head, one pass over the keys it sees with the
// softmax's running maximum and sum.
#include "lba_attn.h"

namespace lba {

int attn_params(const lba_attn& a, AttnParams* p) {
    int rc = check_heads(a.T, a.H, a.D);
    if (rc == LBA_OK) rc = check_heads(a.Tk, a.KV, a.D);
    if (rc == LBA_OK) rc = check_strides(a.q);
    if (rc == LBA_OK) rc = check_strides(a.k);
    if (rc == LBA_OK) rc = check_strides(a.v);
    if (rc == LBA_OK && (a.D < 1 || a.D > 128 || a.count < 0 || a.count > (1 << 20))) rc = LBA_ERR_SHAPE;
    if (rc == LBA_OK && a.H > 0 && (a.KV < 1 || a.H % a.KV != 0)) rc = LBA_ERR_SHAPE;
    if (rc == LBA_OK && !a.starts) {
        if (a.starts_k) rc = LBA_ERR_NULL;
        else if (a.count < 1 ? a.T != 0 || a.Tk != 0 : a.T % a.count != 0 || a.Tk % a.count != 0) rc = LBA_ERR_SHAPE;
    }
    if (rc == LBA_OK) rc = check_float_type(a.type);
    if (rc != LBA_OK) return rc;
    p->starts = a.starts; p->starts_k = a.starts_k ? a.starts_k : a.starts;
    p->q = a.q; p->k = a.k; p->v = a.v;
    p->T = (int32_t)a.T; p->Tk = (int32_t)a.Tk; p->count = (int32_t)a.count;
    p->H = a.H; p->KV = a.KV; p->group = a.KV > 0 ? a.H / a.KV : 1; p->D = a.D;
    p->causal = a.causal != 0; p->clear = a.clear != 0; p->scale = a.scale;
    return LBA_OK;
}

template <typename T, typename TO>
__global__ __launch_bounds__(64) void attn_plain_kernel(AttnParams p) {
    __shared__ float q[128], w[64];
    const int lane = threadIdx.x;
    const int64_t total = (int64_t)p.T * p.H;
    for (int64_t i = blockIdx.x; i < total; i += gridDim.x) {
        const int t = (int)(i / p.H), h = (int)(i % p.H), kv = h / p.group;
        const int b = p.count > 0 ? sequence_of(p.starts, p.T, p.count, t) : -1;
        TO* o = (TO*)p.O + i * p.D;
        if (b < 0) {
            if (p.clear) {
                for (int d = lane; d < p.D; d += 64) store_one(o + d, 0.0f, p.fmt);
                if (p.lse && lane == 0) p.lse[i] = -__builtin_inff();
            }
            continue;
        }
        const Rows rq = rows_of(p.starts, p.T, p.count, b), rk = rows_of(p.starts_k, p.Tk, p.count, b);
        const int seen = p.causal ? max(0, min(rk.n, t - rq.first + rk.n - rq.n + 1)) : rk.n;
        __syncthreads();
        for (int d = lane; d < p.D; d += 64) q[d] = load_one((const T*)p.Q + (int64_t)t * p.q.row + (int64_t)h * p.q.head + d);
        float m = -__builtin_inff(), l = 0.0f, acc0 = 0.0f, acc1 = 0.0f;
        for (int j0 = 0; j0 < seen; j0 += 64) {
            __syncthreads();
            float s = -__builtin_inff();
            if (j0 + lane < seen) {
                const T* k = (const T*)p.K + (int64_t)(rk.first + j0 + lane) * p.k.row + (int64_t)kv * p.k.head;
                s = 0.0f;
                for (int d = 0; d < p.D; ++d) s = fmaf(q[d], load_one(k + d), s);
                s *= p.scale;
            }
            float top = s;
            for (int x = 32; x; x /= 2) top = fmaxf(top, __shfl_xor(top, x));
            top = fmaxf(top, m);
            const float base = top == -__builtin_inff() ? 0.0f : top;
            const float e = j0 + lane < seen ? exp_near(s - base) : 0.0f, f = exp_near(m - base);
            m = top;
            l = l * f + wave_sum(e);
            w[lane] = e;
            __syncthreads();
            acc0 *= f; acc1 *= f;
            const int n = min(64, seen - j0);
            for (int j = 0; j < n; ++j) {
                const T* v = (const T*)p.V + (int64_t)(rk.first + j0 + j) * p.v.row + (int64_t)kv * p.v.head;
                if (lane < p.D) acc0 = fmaf(w[j], load_one(v + lane), acc0);
                if (lane + 64 < p.D) acc1 = fmaf(w[j], load_one(v + lane + 64), acc1);
            }
        }
        const float inv = seen > 0 ? 1.0f / l : 0.0f;
        if (lane < p.D) store_one(o + lane, seen > 0 ? acc0 * inv : 0.0f, p.fmt);
        if (lane + 64 < p.D) store_one(o + lane + 64, seen > 0 ? acc1 * inv : 0.0f, p.fmt);
        if (p.lse && lane == 0) p.lse[i] = seen > 0 ? m + __logf(l) : -__builtin_inff();
    }
}

}  // namespace lba

using namespace lba;

extern "C" int lba_attention(lba_attn a, const void* Q, const void* K, const void* V, void* O, int32_t o_type, lba_infmt o_fmt, float* lse,
                             void* hip_stream) {
    AttnParams p = {};
    int rc = attn_params(a, &p);
    if (rc == LBA_OK) rc = check_out_type(o_type, o_fmt);
    if (rc != LBA_OK) return rc;
    if (p.T == 0 || p.H == 0) return LBA_OK;
    if (!Q || !O || (p.Tk > 0 && (!K || !V))) return LBA_ERR_NULL;
    p.Q = Q; p.K = K; p.V = V; p.O = O; p.lse = lse;
    if (o_type == LBA_CODE8) p.fmt = make_code_fmt(o_fmt);
    const int64_t rows = (int64_t)p.T * p.H;
    const dim3 grid((unsigned)(rows < (1 << 20) ? rows : (1 << 20)));
    const hipStream_t st = (hipStream_t)hip_stream;
#define LBA_ATTN(T) \
    do { \
        if (o_type == LBA_F32) hipLaunchKernelGGL((attn_plain_kernel<T, float>), grid, dim3(64), 0, st, p); \
        else if (o_type == LBA_BF16) hipLaunchKernelGGL((attn_plain_kernel<T, bf16_t>), grid, dim3(64), 0, st, p); \
        else hipLaunchKernelGGL((attn_plain_kernel<T, uint8_t>), grid, dim3(64), 0, st, p); \
    } while (0)
    if (a.type == LBA_F32) LBA_ATTN(float); else LBA_ATTN(bf16_t);
#undef LBA_ATTN
    return hipGetLastError() == hipSuccess ? LBA_OK : LBA_ERR_LAUNCH;
}

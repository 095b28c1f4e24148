// lba_attn_bwd.hip -- the gradients of attention over packed sequences: one wave to a query row of a head (dQ, and the row's sum of G * O), then
// one to a key row of a head of keys, over all the queries that see it.  The weights are made again from lse.
#include "lba_attn.h"

namespace lba {

template <typename T>
__global__ __launch_bounds__(64) void attn_dq_kernel(AttnParams p) {
    __shared__ float q[128], g[128], w[64];
    const int lane = threadIdx.x;
    const int64_t total = (int64_t)p.T * p.H;
    const CodeFmt none = {};
    for (int64_t i = blockIdx.x; i < total; i += gridDim.x) {
        const int t = (int)(i / p.H), h = (int)(i % p.H), kv = h / p.group;
        const int b = p.count > 0 ? sequence_of(p.starts, p.T, p.count, t) : -1;
        T* dq = (T*)p.dQ + (int64_t)t * p.dq.row + (int64_t)h * p.dq.head;
        if (b < 0) {
            if (p.clear)
                for (int d = lane; d < p.D; d += 64) store_one(dq + d, 0.0f, none);
            continue;
        }
        const Rows rq = rows_of(p.starts, p.T, p.count, b), rk = rows_of(p.starts_k, p.Tk, p.count, b);
        const int seen = p.causal ? max(0, min(rk.n, t - rq.first + rk.n - rq.n + 1)) : rk.n;
        __syncthreads();
        float delta = 0.0f;
        for (int d = lane; d < p.D; d += 64) {
            q[d] = load_one((const T*)p.Q + (int64_t)t * p.q.row + (int64_t)h * p.q.head + d);
            g[d] = load_one((const T*)p.G + i * p.D + d);
            delta = fmaf(g[d], load_one((const T*)p.O + i * p.D + d), delta);
        }
        delta = wave_sum(delta);
        if (lane == 0) p.delta[i] = delta;
        const float lse = p.lse[i];
        float acc0 = 0.0f, acc1 = 0.0f;
        for (int j0 = 0; j0 < seen; j0 += 64) {
            __syncthreads();
            float e = 0.0f;
            if (j0 + lane < seen) {
                const T* k = (const T*)p.K + (int64_t)(rk.first + j0 + lane) * p.k.row + (int64_t)kv * p.k.head;
                const T* v = (const T*)p.V + (int64_t)(rk.first + j0 + lane) * p.v.row + (int64_t)kv * p.v.head;
                float s = 0.0f, u = 0.0f;
                for (int d = 0; d < p.D; ++d) { s = fmaf(q[d], load_one(k + d), s); u = fmaf(g[d], load_one(v + d), u); }
                e = exp_near(s * p.scale - lse) * (u - delta);
            }
            w[lane] = e;
            __syncthreads();
            const int n = min(64, seen - j0);
            for (int j = 0; j < n; ++j) {
                const T* k = (const T*)p.K + (int64_t)(rk.first + j0 + j) * p.k.row + (int64_t)kv * p.k.head;
                if (lane < p.D) acc0 = fmaf(w[j], load_one(k + lane), acc0);
                if (lane + 64 < p.D) acc1 = fmaf(w[j], load_one(k + lane + 64), acc1);
            }
        }
        if (lane < p.D) store_one(dq + lane, acc0 * p.scale, none);
        if (lane + 64 < p.D) store_one(dq + lane + 64, acc1 * p.scale, none);
    }
}

template <typename T>
__global__ __launch_bounds__(64) void attn_dkv_kernel(AttnParams p) {
    __shared__ float k[128], v[128], wp[64], ws[64];
    const int lane = threadIdx.x;
    const int64_t total = (int64_t)p.Tk * p.KV;
    const CodeFmt none = {};
    for (int64_t i = blockIdx.x; i < total; i += gridDim.x) {
        const int t = (int)(i / p.KV), kv = (int)(i % p.KV);
        const int b = p.count > 0 ? sequence_of(p.starts_k, p.Tk, p.count, t) : -1;
        T* dk = (T*)p.dK + (int64_t)t * p.dk.row + (int64_t)kv * p.dk.head;
        T* dv = (T*)p.dV + (int64_t)t * p.dv.row + (int64_t)kv * p.dv.head;
        if (b < 0) {
            if (p.clear)
                for (int d = lane; d < p.D; d += 64) { store_one(dk + d, 0.0f, none); store_one(dv + d, 0.0f, none); }
            continue;
        }
        const Rows rq = rows_of(p.starts, p.T, p.count, b), rk = rows_of(p.starts_k, p.Tk, p.count, b);
        const int first = p.causal ? min(rq.n, max(0, t - rk.first - (rk.n - rq.n))) : 0;
        __syncthreads();
        for (int d = lane; d < p.D; d += 64) {
            k[d] = load_one((const T*)p.K + (int64_t)t * p.k.row + (int64_t)kv * p.k.head + d);
            v[d] = load_one((const T*)p.V + (int64_t)t * p.v.row + (int64_t)kv * p.v.head + d);
        }
        float dk0 = 0.0f, dk1 = 0.0f, dv0 = 0.0f, dv1 = 0.0f;
        for (int h = kv * p.group; h < (kv + 1) * p.group; ++h) {
            for (int i0 = first; i0 < rq.n; i0 += 64) {
                __syncthreads();
                float e = 0.0f, f = 0.0f;
                if (i0 + lane < rq.n) {
                    const int64_t at = (int64_t)(rq.first + i0 + lane);
                    const T* q = (const T*)p.Q + at * p.q.row + (int64_t)h * p.q.head;
                    const T* g = (const T*)p.G + (at * p.H + h) * p.D;
                    float s = 0.0f, u = 0.0f;
                    for (int d = 0; d < p.D; ++d) { s = fmaf(k[d], load_one(q + d), s); u = fmaf(v[d], load_one(g + d), u); }
                    e = exp_near(s * p.scale - p.lse[at * p.H + h]);
                    f = e * (u - p.delta[at * p.H + h]);
                }
                wp[lane] = e;
                ws[lane] = f;
                __syncthreads();
                const int n = min(64, rq.n - i0);
                for (int j = 0; j < n; ++j) {
                    const int64_t at = (int64_t)(rq.first + i0 + j);
                    const T* q = (const T*)p.Q + at * p.q.row + (int64_t)h * p.q.head;
                    const T* g = (const T*)p.G + (at * p.H + h) * p.D;
                    if (lane < p.D) { dk0 = fmaf(ws[j], load_one(q + lane), dk0); dv0 = fmaf(wp[j], load_one(g + lane), dv0); }
                    if (lane + 64 < p.D) { dk1 = fmaf(ws[j], load_one(q + lane + 64), dk1); dv1 = fmaf(wp[j], load_one(g + lane + 64), dv1); }
                }
            }
        }
        if (lane < p.D) { store_one(dk + lane, dk0 * p.scale, none); store_one(dv + lane, dv0, none); }
        if (lane + 64 < p.D) { store_one(dk + lane + 64, dk1 * p.scale, none); store_one(dv + lane + 64, dv1, none); }
    }
}

}  // namespace lba

using namespace lba;

extern "C" {

size_t lba_attention_bwd_workspace_bytes(int64_t T, int64_t H) {
    if (check_heads(T, H, 1) != LBA_OK) return 0;
    return align256((size_t)T * (size_t)H * sizeof(float));
}

int lba_attention_bwd(lba_attn a, const void* G, const void* Q, const void* K, const void* V, const void* O, const float* lse, void* dQ,
                      lba_strides dq_at, void* dK, lba_strides dk_at, void* dV, lba_strides dv_at, void* workspace, size_t workspace_bytes,
                      void* hip_stream) {
    AttnParams p = {};
    int rc = attn_params(a, &p);
    if (rc == LBA_OK) rc = check_strides(dq_at);
    if (rc == LBA_OK) rc = check_strides(dk_at);
    if (rc == LBA_OK) rc = check_strides(dv_at);
    if (rc != LBA_OK) return rc;
    const bool queries = p.T > 0 && p.H > 0, keys = p.Tk > 0 && p.KV > 0;
    if (!queries && !keys) return LBA_OK;
    if ((queries && (!G || !Q || !O || !lse || !dQ || !workspace)) || (keys && (!K || !V || !dK || !dV))) return LBA_ERR_NULL;
    if (queries && (uintptr_t)workspace % 256 != 0) return LBA_ERR_ALIGN;
    if (workspace_bytes < lba_attention_bwd_workspace_bytes(p.T, p.H)) return LBA_ERR_SHAPE;
    p.Q = Q; p.K = K; p.V = V; p.O = (void*)O; p.G = G; p.lse = (float*)lse; p.delta = (float*)workspace;
    p.dQ = dQ; p.dK = dK; p.dV = dV; p.dq = dq_at; p.dk = dk_at; p.dv = dv_at;
    const hipStream_t st = (hipStream_t)hip_stream;
    const int64_t nq = (int64_t)p.T * p.H, nk = (int64_t)p.Tk * p.KV;
    const dim3 gq((unsigned)(nq < (1 << 20) ? nq : (1 << 20))), gk((unsigned)(nk < (1 << 20) ? nk : (1 << 20)));
    if (queries) {
        if (a.type == LBA_F32) hipLaunchKernelGGL((attn_dq_kernel<float>), gq, dim3(64), 0, st, p);
        else hipLaunchKernelGGL((attn_dq_kernel<bf16_t>), gq, dim3(64), 0, st, p);
    }
    if (keys) {
        if (a.type == LBA_F32) hipLaunchKernelGGL((attn_dkv_kernel<float>), gk, dim3(64), 0, st, p);
        else hipLaunchKernelGGL((attn_dkv_kernel<bf16_t>), gk, dim3(64), 0, st, p);
    }
    return hipGetLastError() == hipSuccess ? LBA_OK : LBA_ERR_LAUNCH;
}

}  // extern "C"

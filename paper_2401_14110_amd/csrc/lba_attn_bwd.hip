// lba_attn_bwd.hip -- the gradients of attention over packed sequences: the join of parts, entry points.
#include "lba_attn_tile.h"

namespace lba {

// Gradients from the parts: a workgroup a row, a lane an element of its heads.  KEYS: dK, and blockIdx.y == 1: dV; else dQ.
template <typename T, bool KEYS> __global__ __launch_bounds__(256) void attn_join_grad_kernel(AttnParams p) {
    const int heads = KEYS ? p.KV : p.H, total = KEYS ? p.Tk : p.T;
    const int64_t all = (int64_t)total * heads * p.D;
    const float* part = p.part + blockIdx.y * p.slices * all;
    T* out = (T*)(!KEYS ? p.dQ : blockIdx.y ? p.dV : p.dK);
    const lba_strides at = !KEYS ? p.dq : blockIdx.y ? p.dv : p.dk;
    const CodeFmt none = {};
    for (int t = blockIdx.x; t < total; t += gridDim.x) {
        const int b = KEYS ? sequence_of(p.starts_k, p.Tk, p.count, t) : sequence_of(p.starts, p.T, p.count, t);
        if (b < 0) continue;
        const Rows rq = rows_of(p.starts, p.T, p.count, b), rk = rows_of(p.starts_k, p.Tk, p.count, b);
        const int steps = KEYS ? steps_of_keys(p, rq, rk, (t - rk.first) / kTileRows, kStep<T>) * p.group : steps_of_queries(p, rq, rk, (t - rq.first) / kTileRows, kStep<T>);
        const int n = slices_used(steps, p.slices);
        if (n <= 1) continue;                            // stored by its only workgroup
        for (int i = threadIdx.x; i < heads * p.D; i += 256) {
            float v = 0.0f;
            for (int x = 0; x < n; ++x) v += part[x * all + (int64_t)t * heads * p.D + i];
            store_one(out + (int64_t)t * at.row + (int64_t)(i / p.D) * at.head + i % p.D, v, none);
        }
    }
}
template <typename T, bool KEYS> static void launch_join_grad(const AttnParams& p, hipStream_t st) {
    const int rows = KEYS ? p.Tk : p.T;
    hipLaunchKernelGGL((attn_join_grad_kernel<T, KEYS>), dim3((unsigned)(rows < (1 << 20) ? rows : (1 << 20)), KEYS ? 2 : 1), dim3(256), 0, st, p);
}

}  // namespace lba

using namespace lba;

extern "C" {

size_t lba_attention_bwd_workspace_bytes(lba_attn a) {
    AttnParams p = {};
    AttnPlan plan;
    if (attn_params(a, &p) != LBA_OK || attn_plan(a, &plan) != LBA_OK) return 0;
    const size_t delta = align256((size_t)p.T * (size_t)p.H * sizeof(float));
    const size_t dq = plan.slices_dq > 1 ? (size_t)plan.slices_dq * (size_t)p.T * (size_t)p.H : 0;
    const size_t dkv = plan.slices_dkv > 1 ? (size_t)plan.slices_dkv * (size_t)p.Tk * (size_t)p.KV * 2 : 0;
    return delta + align256((dq > dkv ? dq : dkv) * (size_t)p.D * sizeof(float));       // one after the other in the same place
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
    if (workspace_bytes < lba_attention_bwd_workspace_bytes(a)) return LBA_ERR_SHAPE;
    p.Q = Q; p.K = K; p.V = V; p.O = (void*)O; p.G = G; p.lse = (float*)lse; p.delta = (float*)workspace;
    p.dQ = dQ; p.dK = dK; p.dV = dV; p.dq = dq_at; p.dk = dk_at; p.dv = dv_at;
    const hipStream_t st = (hipStream_t)hip_stream;
    AttnPlan plan;
    rc = attn_plan(a, &plan);
    if (rc != LBA_OK) return rc;
    p.part = (float*)((char*)workspace + align256((size_t)p.T * (size_t)p.H * sizeof(float)));
    const int64_t size = a.type == LBA_F32 ? 4 : 2;
    if (queries && (plan.tiles_q > 0 || p.clear)) {
        const bool direct = whole_pieces(K, a.k, a.D, size) && whole_pieces(V, a.v, a.D, size);
        p.tiles = (int32_t)plan.tiles_q;
        p.units = (int32_t)(plan.tiles_q * p.H);
        p.slices = plan.slices_dq;
        if (a.type == LBA_F32) launch_attn_dq<float>(p, direct, st); else launch_attn_dq<bf16_t>(p, direct, st);
        if (p.slices > 1) { if (a.type == LBA_F32) launch_join_grad<float, false>(p, st); else launch_join_grad<bf16_t, false>(p, st); }
    }
    if (keys && (plan.tiles_k > 0 || p.clear)) {
        const lba_strides g = {(int64_t)a.H * a.D, a.D};
        const bool direct = whole_pieces(Q, a.q, a.D, size) && whole_pieces(G, g, a.D, size);
        p.tiles = (int32_t)plan.tiles_k;
        p.units = (int32_t)(plan.tiles_k * p.KV);
        p.slices = plan.slices_dkv;
        if (a.type == LBA_F32) launch_attn_dkv<float>(p, direct, st); else launch_attn_dkv<bf16_t>(p, direct, st);
        if (p.slices > 1) { if (a.type == LBA_F32) launch_join_grad<float, true>(p, st); else launch_join_grad<bf16_t, true>(p, st); }
    }
    return hipGetLastError() == hipSuccess ? LBA_OK : LBA_ERR_LAUNCH;
}

}  // extern "C"

// lba_attn_bwd.hip -- the gradients of attention over packed sequences: the join of parts, entry points.
#include "lba_attn_tile.h"

namespace lba {

// Gradients from the parts: a workgroup eight heads of a row, a wave two, a lane two elements.  KEYS: dK, and blockIdx.z == 1: dV; else dQ.
template <typename T, bool KEYS> __global__ __launch_bounds__(256) void attn_join_grad_kernel(AttnParams p) {
    const int heads = KEYS ? p.KV : p.H, total = KEYS ? p.Tk : p.T;
    const int64_t all = (int64_t)total * heads * p.D;
    const float* part = p.part + blockIdx.z * p.slices * all;
    T* out = (T*)(!KEYS ? p.dQ : blockIdx.z ? p.dV : p.dK);
    const lba_strides at = !KEYS ? p.dq : blockIdx.z ? p.dv : p.dk;
    const CodeFmt none = {};
    for (int t = blockIdx.x; t < total; t += gridDim.x) {
        const TileOf own = KEYS ? find_row(p.starts_k, p.Tk, p.starts, p.T, p.count, t) : find_row(p.starts, p.T, p.starts_k, p.Tk, p.count, t);
        if (own.b < 0) continue;
        const Rows rq = KEYS ? own.other : own.mine, rk = KEYS ? own.mine : own.other;
        const int steps = KEYS ? steps_of_keys(p, rq, rk, (t - rk.first) / kTileRows, kStep<T>) * p.group : steps_of_queries(p, rq, rk, (t - rq.first) / kTileRows, kStep<T>);
        const int n = slices_used(steps, p.slices);
        if (n <= 1) continue;                            // stored by its only workgroup
        const int h0 = blockIdx.y * 8 + threadIdx.x / 64 * 2, lane = threadIdx.x & 63, some = min(2, heads - h0);
        if (some < 1) return;
        float v[2][2];
        sum_parts(part + ((int64_t)t * heads + h0) * p.D, all, n, some, p.D, [](int, int) { return 1.0f; }, v);
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int i = 0; i < 2; ++i)
                if (h < some && lane + 64 * i < p.D) store_one(out + (int64_t)t * at.row + (int64_t)(h0 + h) * at.head + lane + 64 * i, v[h][i], none);
    }
}
template <typename T, bool KEYS> static void launch_join_grad(const AttnParams& p, hipStream_t st) {
    const int rows = KEYS ? p.Tk : p.T, heads = KEYS ? p.KV : p.H;
    hipLaunchKernelGGL((attn_join_grad_kernel<T, KEYS>), dim3((unsigned)(rows < (1 << 20) ? rows : (1 << 20)), (unsigned)(heads + 7) / 8, KEYS ? 2 : 1), dim3(256), 0, st, p);
}

}  // namespace lba

using namespace lba;

extern "C" {

size_t lba_attention_bwd_workspace_bytes(lba_attn a) {
    AttnParams p = {};
    take_fine(&a.type);
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
    const bool fine = take_fine(&a.type);
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
    p.fine = fine;
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

// lba_attn_bwd.hip -- the gradients of attention over packed sequences: entry points.
#include "lba_attn_tile.h"

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
    }
    if (keys && (plan.tiles_k > 0 || p.clear)) {
        const lba_strides g = {(int64_t)a.H * a.D, a.D};
        const bool direct = whole_pieces(Q, a.q, a.D, size) && whole_pieces(G, g, a.D, size);
        p.tiles = (int32_t)plan.tiles_k;
        p.units = (int32_t)(plan.tiles_k * p.KV);
        p.slices = plan.slices_dkv;
        if (a.type == LBA_F32) launch_attn_dkv<float>(p, direct, st); else launch_attn_dkv<bf16_t>(p, direct, st);
    }
    return hipGetLastError() == hipSuccess ? LBA_OK : LBA_ERR_LAUNCH;
}

}  // extern "C"

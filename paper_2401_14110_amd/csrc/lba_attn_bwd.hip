// lba_attn_bwd.hip -- the gradients of attention over packed sequences: entry points.
#include "lba_attn_tile.h"

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
    const int64_t tiles_q = most_tiles(p.starts, p.T, p.count, kTileRows), tiles_k = most_tiles(p.starts_k, p.Tk, p.count, kTileRows);
    if (tiles_q * p.H > kMostUnits || tiles_k * p.KV > kMostUnits) return LBA_ERR_SHAPE;
    const int64_t size = a.type == LBA_F32 ? 4 : 2;
    if (queries && (tiles_q > 0 || p.clear)) {
        const bool direct = whole_pieces(K, a.k, a.D, size) && whole_pieces(V, a.v, a.D, size);
        p.tiles = (int32_t)tiles_q;
        p.units = (int32_t)(tiles_q * p.H);
        if (a.type == LBA_F32) launch_attn_dq<float>(p, direct, st); else launch_attn_dq<bf16_t>(p, direct, st);
    }
    if (keys && (tiles_k > 0 || p.clear)) {
        const lba_strides g = {(int64_t)a.H * a.D, a.D};
        const bool direct = whole_pieces(Q, a.q, a.D, size) && whole_pieces(G, g, a.D, size);
        p.tiles = (int32_t)tiles_k;
        p.units = (int32_t)(tiles_k * p.KV);
        if (a.type == LBA_F32) launch_attn_dkv<float>(p, direct, st); else launch_attn_dkv<bf16_t>(p, direct, st);
    }
    return hipGetLastError() == hipSuccess ? LBA_OK : LBA_ERR_LAUNCH;
}

}  // extern "C"

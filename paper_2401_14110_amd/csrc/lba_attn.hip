// lba_attn.hip -- attention over packed sequences: the description's checks, how passes are cut into parts and the join of the forward pass's, its
// entry point.
#include "lba_attn_tile.h"

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

// With few workgroups the steps of each are cut into parts, whose sums are joined by a launch of their own: so many that the card is full, but parts
// of `least` steps at least of an average sequence.
static int slices_for(int64_t units, int64_t steps, int64_t slots, int64_t least) {
    if (units < 1) return 1;
    int64_t n = slots / units;
    if (n > steps / least) n = steps / least;
    return (int)(n < 1 ? 1 : n > kMostSlices ? kMostSlices : n);
}

int attn_plan(const lba_attn& a, AttnPlan* plan) {
    plan->tiles_q = most_tiles(a.starts, a.T, a.count, kTileRows);
    plan->tiles_k = most_tiles(a.starts_k ? a.starts_k : a.starts, a.Tk, a.count, kTileRows);
    if (plan->tiles_q * a.H > kMostUnits || plan->tiles_k * a.KV > kMostUnits) return LBA_ERR_SHAPE;
    const int64_t step = a.type == LBA_F32 ? 32 : 64, count = a.count > 0 ? a.count : 1;
    const int64_t keys = a.Tk / count / step, queries = a.T / count / step * (a.KV > 0 ? a.H / a.KV : 1);
    // Bfloat16: two workgroups a CU, which is what the 256 have room for, of dK and dV with heads above 64 one; the tiles counted are those that there may be.
    // Float32's steps of half as many rows take three times as long, so shorter parts are worth a join.  Its numbers of workgroups are those that took least
    // for 7 sequences of 33 to 517, 6 heads of 83, where a seventh of the tiles are empty; with 384, 512 and 1024: forward (two on a CU) 35, 31 and 30 us, dQ
    // (one) 51, 61 and 72, dK and dV (one) 64, 60 and 59, their join 11, 12 and 13.
    const bool f32 = a.type == LBA_F32;
    const int64_t least = f32 ? 2 : 4;
    plan->slices = slices_for(plan->tiles_q * a.H, keys, f32 ? 1024 : 512, least);
    plan->slices_dq = slices_for(plan->tiles_q * a.H, keys, f32 ? 384 : 512, least);
    plan->slices_dkv = slices_for(plan->tiles_k * a.KV, queries, f32 || a.D <= 64 ? 512 : 256, least);
    return LBA_OK;
}

// O and lse from the parts: a workgroup eight heads of a row, a wave two, a lane a part's weight and then two elements.
template <typename T> __global__ __launch_bounds__(256) void attn_join_kernel(AttnParams p) {
    const int64_t rows = (int64_t)p.T * p.H;
    const int lane = threadIdx.x & 63;
    for (int t = blockIdx.x; t < p.T; t += gridDim.x) {
        const TileOf at = find_row(p.starts, p.T, p.starts_k, p.Tk, p.count, t);
        if (at.b < 0) continue;
        const Rows rq = at.mine, rk = at.other;
        const int n = slices_used(steps_of_queries(p, rq, rk, (t - rq.first) / kTileRows, kStep<T>), p.slices);
        if (n <= 1) continue;                            // stored by its only workgroup
        const int h0 = blockIdx.y * 8 + threadIdx.x / 64 * 2, heads = min(2, p.H - h0);
        if (heads < 1) return;
        const int64_t row = (int64_t)t * p.H + h0;
        float most[2], weight[2], sum[2], v[2][2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const float* end = p.part + p.slices * rows * p.D + (min(lane, n - 1) * rows + row + (h < heads ? h : 0)) * 2;
            most[h] = end[0];
            sum[h] = end[1];
        }
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const float top = wave_max(most[h]), base = top == -__builtin_inff() ? 0.0f : top;
            weight[h] = __builtin_amdgcn_exp2f(most[h] - base);
            sum[h] = wave_sum(lane < n ? weight[h] * sum[h] : 0.0f);
            most[h] = top;
        }
        sum_parts(p.part + row * p.D, rows * p.D, n, heads, p.D, [&](int h, int x) { return __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(weight[h]), x)); }, v);
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            if (h >= heads) break;
            const float inv = sum[h] == 0.0f ? 0.0f : 1.0f / sum[h];
            with_output(p, [&](auto* o) {
#pragma unroll
                for (int i = 0; i < 2; ++i)
                    if (lane + 64 * i < p.D) store_one(o + (row + h) * p.D + lane + 64 * i, v[h][i] * inv, p.fmt);
            });
            if (p.lse && lane == 0) p.lse[row + h] = sum[h] == 0.0f ? -__builtin_inff() : (most[h] + __builtin_amdgcn_logf(sum[h])) * 0.693147181f;
        }
    }
}

template <typename T> static void launch_join(const AttnParams& p, hipStream_t st) {
    hipLaunchKernelGGL((attn_join_kernel<T>), dim3((unsigned)(p.T < (1 << 20) ? p.T : (1 << 20)), (unsigned)(p.H + 7) / 8), dim3(256), 0, st, p);
}

}  // namespace lba

using namespace lba;

extern "C" {

size_t lba_attention_workspace_bytes(lba_attn a) {
    AttnParams p = {};
    take_fine(&a.type);
    AttnPlan plan;
    if (attn_params(a, &p) != LBA_OK || attn_plan(a, &plan) != LBA_OK || plan.slices == 1) return 0;
    return align256((size_t)plan.slices * (size_t)p.T * (size_t)p.H * (size_t)(p.D + 2) * sizeof(float));
}

int lba_attention(lba_attn a, const void* Q, const void* K, const void* V, void* O, int32_t o_type, lba_infmt o_fmt, float* lse, void* workspace,
                  size_t workspace_bytes, void* hip_stream) {
    AttnParams p = {};
    const bool fine = take_fine(&a.type);
    int rc = attn_params(a, &p);
    if (rc == LBA_OK) rc = check_out_type(o_type, o_fmt);
    if (rc != LBA_OK) return rc;
    if (p.T == 0 || p.H == 0) return LBA_OK;
    if (!Q || !O || (p.Tk > 0 && (!K || !V))) return LBA_ERR_NULL;
    p.Q = Q; p.K = K; p.V = V; p.O = O; p.lse = lse;
    if (o_type == LBA_CODE8) p.fmt = make_code_fmt(o_fmt);
    p.o_type = o_type; p.fine = fine || o_type == LBA_F32;
    AttnPlan plan;
    rc = attn_plan(a, &plan);
    if (rc != LBA_OK) return rc;
    p.tiles = (int32_t)plan.tiles_q;
    p.units = (int32_t)(plan.tiles_q * p.H);
    p.slices = plan.slices;
    if (p.units == 0 && !p.clear) return LBA_OK;
    if (p.slices > 1) {
        if (!workspace) return LBA_ERR_NULL;
        if ((uintptr_t)workspace % 256 != 0) return LBA_ERR_ALIGN;
        if (workspace_bytes < lba_attention_workspace_bytes(a)) return LBA_ERR_SHAPE;
        p.part = (float*)workspace;
    }
    const int64_t size = a.type == LBA_F32 ? 4 : 2;
    const bool direct = whole_pieces(K, a.k, a.D, size) && whole_pieces(V, a.v, a.D, size);
    const hipStream_t st = (hipStream_t)hip_stream;
    if (a.type == LBA_F32) launch_attn<float>(p, direct, st); else launch_attn<bf16_t>(p, direct, st);
    if (p.slices > 1) { if (a.type == LBA_F32) launch_join<float>(p, st); else launch_join<bf16_t>(p, st); }
    return hipGetLastError() == hipSuccess ? LBA_OK : LBA_ERR_LAUNCH;
}

}  // extern "C"

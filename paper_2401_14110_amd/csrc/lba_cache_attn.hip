// lba_cache_attn.hip -- attention over the cache: how it is cut, the join of the chunks, entry points.
#include "lba_cache_attn.h"

namespace lba {

template <typename T> void launch_cache_attn(const CacheAttnParams& p, int r, hipStream_t st);

// Row `out` of O from its chunks: a workgroup a row, a group of lanes for every piece of four elements, chunks in turn over the groups.
template <typename TO> __global__ __launch_bounds__(256) void cache_join_kernel(CacheAttnParams p, int rows_of_tile) {
    __shared__ float weight[256];
    __shared__ f32x4_c sums[256];
    __shared__ float parts[4];
    const int64_t out = blockIdx.x;
    const int D = p.c.D, h = (int)(out % p.H);
    const int64_t token = out / p.H;
    const int b = (int)(token / p.fresh), r = (int)(token % p.fresh) * p.group + h % p.group, rows = p.fresh * p.group;
    const int seen = row_seen(p, b, min(r / rows_of_tile * rows_of_tile + rows_of_tile, rows) - 1);
    const int n = (seen + p.chunk - 1) / p.chunk;
    if (n <= 1) return;                                  // stored by its only workgroup
    const float* part = p.part + out * p.chunks * D;
    const float* end = p.part + (int64_t)p.c.count * p.fresh * p.H * p.chunks * D + out * p.chunks * 2;
    const int lane = threadIdx.x & 63, wave = threadIdx.x / 64;
    float m = -__builtin_inff();
    for (int i = threadIdx.x; i < n; i += 256) m = fmaxf(m, end[2 * i]);
#pragma unroll
    for (int x = 32; x; x /= 2) m = fmaxf(m, __shfl_xor(m, x));
    if (lane == 0) parts[wave] = m;
    __syncthreads();
    m = fmaxf(fmaxf(parts[0], parts[1]), fmaxf(parts[2], parts[3]));
    const int pieces = D / 4, groups = 256 / pieces, g = (int)threadIdx.x / pieces, piece = (int)threadIdx.x % pieces;
    f32x4_c v = {0.0f, 0.0f, 0.0f, 0.0f};
    float l = 0.0f;
    for (int i0 = 0; i0 < n; i0 += 256) {
        __syncthreads();
        const int i = i0 + (int)threadIdx.x;
        const float w = i < n && m != -__builtin_inff() ? __builtin_amdgcn_exp2f(end[2 * i] - m) : 0.0f;
        weight[threadIdx.x] = w;
        if (i < n) l = fmaf(w, end[2 * i + 1], l);
        __syncthreads();
        if (g < groups)
            for (int k = g; k < 256 && i0 + k < n; k += groups) v += weight[k] * *(const f32x4_c*)&part[(int64_t)(i0 + k) * D + piece * 4];
    }
    l = wave_sum(l);
    __syncthreads();
    if (lane == 0) parts[wave] = l;
    sums[threadIdx.x] = v;
    __syncthreads();
    if (g != 0) return;
    l = (parts[0] + parts[1]) + (parts[2] + parts[3]);
    for (int x = 1; x < groups; ++x) v += sums[x * pieces + piece];
    const float inv = l == 0.0f ? 0.0f : 1.0f / l;
    const float o[4] = {v[0] * inv, v[1] * inv, v[2] * inv, v[3] * inv};
    store_vec<4>((TO*)p.O + out * D + piece * 4, o, p.fmt);
}

// How the rows and positions are cut: rows of a tile, and a chunk's positions, so many that there are about 2048 workgroups where every
// sequence fills its table (four on every CU twice), and 256 at least (two steps of each wave).
struct CachePlan {
    int32_t r, row_tiles;
    int64_t chunk, chunks, rows;
};
static int cache_plan(int64_t count, int64_t table_row, int64_t page, int64_t fresh, int64_t H, int64_t KV, CachePlan* c) {
    const int64_t room = table_row * page, rows = fresh * (H / KV);
    c->r = rows > 16 ? 2 : 1;
    const int64_t row_tiles = (rows + 16 * c->r - 1) / (16 * c->r), units = count * KV * row_tiles;
    if (room > (1 << 30) || KV * row_tiles > 65535 || count > 65535) return LBA_ERR_SHAPE;
    c->row_tiles = (int32_t)row_tiles;
    c->chunk = (room * units + 2047) / 2048;
    c->chunk = (c->chunk + 127) / 128 * 128;
    if (c->chunk < 256) c->chunk = 256;
    c->chunks = room > c->chunk ? (room + c->chunk - 1) / c->chunk : 1;
    c->rows = count * fresh * H;
    return c->chunks * units < (1 << 24) && c->rows < (1 << 24) ? LBA_OK : LBA_ERR_SHAPE;
}

}  // namespace lba

using namespace lba;

extern "C" {

size_t lba_cache_attention_workspace_bytes(int64_t count, int64_t table_row, int32_t page, int64_t fresh, int64_t H, int32_t KV, int32_t D) {
    CachePlan c;
    if (count < 1 || table_row < 0 || page < 1 || fresh < 1 || H < 1 || KV < 1 || H % KV != 0 || count > (1 << 20) || table_row > 2147483647LL || page > 65536 ||
        fresh > 2147483647LL / (count * H) || cache_plan(count, table_row, page, fresh, H, KV, &c) != LBA_OK || c.chunks == 1)
        return 0;
    return align256((size_t)c.rows * (size_t)c.chunks * (size_t)(D + 2) * sizeof(float));
}

int lba_cache_attention(lba_cache4 c, const void* Q, lba_strides q_at, int32_t type, int64_t fresh, int64_t H, float scale, void* O, int32_t o_type,
                        lba_infmt o_fmt, void* workspace, size_t workspace_bytes, void* hip_stream) {
    CacheAttnParams p = {};
    int rc = cache_params(c, &p.c);
    if (rc == LBA_OK) rc = check_strides(q_at);
    if (rc == LBA_OK && (fresh < 0 || fresh > 2147483647LL || H < 0 || H > 65535 || (H > 0 && (c.KV < 1 || H % c.KV != 0)))) rc = LBA_ERR_SHAPE;
    if (rc == LBA_OK && (c.count * H > 0 && fresh > 2147483647LL / (c.count * H))) rc = LBA_ERR_SHAPE;
    if (rc == LBA_OK) rc = check_float_type(type);
    if (rc == LBA_OK) rc = check_out_type(o_type, o_fmt);
    if (rc != LBA_OK) return rc;
    if (c.count == 0 || fresh == 0 || H == 0) return LBA_OK;
    const bool lines = c.table_row > 0 && c.pages > 0;
    if (!Q || !O || !c.lens || (c.table_row > 0 && !c.table) || (lines && (!c.k || !c.k_scale || !c.v || !c.v_scale))) return LBA_ERR_NULL;
    CachePlan plan;
    if (cache_plan(c.count, c.table_row, c.page, fresh, H, c.KV, &plan) != LBA_OK) return LBA_ERR_SHAPE;
    const size_t need = lba_cache_attention_workspace_bytes(c.count, c.table_row, c.page, fresh, H, c.KV, c.D);
    if (need > 0) {
        if (!workspace) return LBA_ERR_NULL;
        if ((uintptr_t)workspace % 256 != 0) return LBA_ERR_ALIGN;
        if (workspace_bytes < need) return LBA_ERR_SHAPE;
    }
    p.Q = Q; p.O = O; p.q = q_at; p.fresh = (int32_t)fresh; p.H = (int32_t)H; p.group = (int32_t)(H / c.KV); p.scale = scale;
    if (o_type == LBA_CODE8) p.fmt = make_code_fmt(o_fmt);
    p.o_type = o_type; p.part = (float*)workspace; p.room = (int32_t)(c.table_row * c.page);
    if (!lines) p.room = 0;                              // nothing is held anywhere
    p.chunk = (int32_t)plan.chunk; p.chunks = (int32_t)plan.chunks; p.row_tiles = plan.row_tiles;
    const hipStream_t st = (hipStream_t)hip_stream;
    if (type == LBA_F32) launch_cache_attn<float>(p, plan.r, st); else launch_cache_attn<bf16_t>(p, plan.r, st);
    if (plan.chunks > 1) {
        const dim3 grid((unsigned)plan.rows);
        if (o_type == LBA_F32) hipLaunchKernelGGL((cache_join_kernel<float>), grid, dim3(256), 0, st, p, 16 * plan.r);
        else if (o_type == LBA_BF16) hipLaunchKernelGGL((cache_join_kernel<bf16_t>), grid, dim3(256), 0, st, p, 16 * plan.r);
        else hipLaunchKernelGGL((cache_join_kernel<uint8_t>), grid, dim3(256), 0, st, p, 16 * plan.r);
    }
    return hipGetLastError() == hipSuccess ? LBA_OK : LBA_ERR_LAUNCH;
}

}  // extern "C"

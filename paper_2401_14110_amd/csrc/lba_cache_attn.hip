// lba_cache_attn.hip -- attention over the cache: how it is cut, the join of the chunks, entry points.
#include "lba_cache_attn.h"

namespace lba {

// where row `out` of O has its chunks, and how many there are
__device__ __forceinline__ int chunks_of_row(const CacheAttnParams& p, int64_t out, int rows_of_tile) {
    const int64_t token = out / p.H;
    const int b = (int)(token / p.fresh), r = (int)(token % p.fresh) * p.group + (int)(out % p.H) % p.group, rows = p.fresh * p.group;
    return (row_seen(p, b, min(r / rows_of_tile * rows_of_tile + rows_of_tile, rows) - 1) + p.chunk - 1) / p.chunk;
}
__device__ __forceinline__ const float* ends_of_row(const CacheAttnParams& p, int64_t out) {
    return p.part + (int64_t)p.c.count * p.fresh * p.H * p.chunks * p.c.D + out * p.chunks * 2;
}
__device__ __forceinline__ void store_joined(const CacheAttnParams& p, int64_t at, f32x4_c v, float l) {
    const float inv = l == 0.0f ? 0.0f : 1.0f / l;
    const float o[4] = {v[0] * inv, v[1] * inv, v[2] * inv, v[3] * inv};
    if (p.o_type == LBA_F32) store_vec<4>((float*)p.O + at, o, p.fmt);
    else if (p.o_type == LBA_BF16) store_vec<4>((bf16_t*)p.O + at, o, p.fmt);
    else store_vec<4>((uint8_t*)p.O + at, o, p.fmt);
}

// Few chunks a row: D / 4 lanes take a row, each its four elements of every chunk.
__global__ __launch_bounds__(256) void cache_join_few_kernel(CacheAttnParams p, int rows_of_tile, int64_t rows) {
    const int pieces = p.c.D / 4, per = 256 / pieces, piece = (int)threadIdx.x % pieces;
    const int64_t out = (int64_t)blockIdx.x * per + (int)threadIdx.x / pieces;
    if ((int)threadIdx.x / pieces >= per || out >= rows) return;
    const int n = chunks_of_row(p, out, rows_of_tile);
    if (n <= 1) return;                                  // stored by its only workgroup
    const float* end = ends_of_row(p, out);
    const float* part = p.part + out * p.chunks * p.c.D + piece * 4;
    float m = -__builtin_inff(), l = 0.0f;
    for (int i = 0; i < n; ++i) m = fmaxf(m, end[2 * i]);
    const float base = m == -__builtin_inff() ? 0.0f : m;            // (all scores -infinity: weights of 0; all NaN, which no maximum is: sums of NaN)
    f32x4_c v = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll 4
    for (int i = 0; i < n; ++i) {
        const float w = __builtin_amdgcn_exp2f(end[2 * i] - base);
        l = fmaf(w, end[2 * i + 1], l);
        v += w * *(const f32x4_c*)&part[(int64_t)i * p.c.D];
    }
    store_joined(p, out * p.c.D + piece * 4, v, l);
}

// Many: row blockIdx.x, elements 32 blockIdx.y ..: eight lanes for the 32 elements, the chunks in turn over the 32 groups of lanes.
__global__ __launch_bounds__(256) void cache_join_kernel(CacheAttnParams p, int rows_of_tile) {
    __shared__ float weight[256];
    __shared__ f32x4_c sums[4][8];
    __shared__ float parts[4];
    const int64_t out = blockIdx.x;
    const int n = chunks_of_row(p, out, rows_of_tile);
    if (n <= 1) return;
    const int D = p.c.D, lane = threadIdx.x & 63, wave = threadIdx.x / 64, g = (int)threadIdx.x / 8, piece = (int)threadIdx.x % 8;
    const float* part = p.part + out * p.chunks * D + blockIdx.y * 32 + piece * 4;
    const float* end = ends_of_row(p, out);
    float m = -__builtin_inff();
    for (int i = threadIdx.x; i < n; i += 256) m = fmaxf(m, end[2 * i]);
#pragma unroll
    for (int x = 32; x; x /= 2) m = fmaxf(m, __shfl_xor(m, x));
    if (lane == 0) parts[wave] = m;
    __syncthreads();
    m = fmaxf(fmaxf(parts[0], parts[1]), fmaxf(parts[2], parts[3]));
    f32x4_c v = {0.0f, 0.0f, 0.0f, 0.0f};
    float l = 0.0f;
    for (int i0 = 0; i0 < n; i0 += 256) {
        __syncthreads();
        const int i = i0 + (int)threadIdx.x;
        const float w = i < n && m != -__builtin_inff() ? __builtin_amdgcn_exp2f(end[2 * i] - m) : 0.0f;
        weight[threadIdx.x] = w;
        if (i < n) l = fmaf(w, end[2 * i + 1], l);
        __syncthreads();
#pragma unroll
        for (int k = 0; k < 8; ++k) {                    // chunks that are not there: the first one's, with no weight
            const int at = g + 32 * k;
            const f32x4_c x = *(const f32x4_c*)&part[(int64_t)(i0 + at < n ? i0 + at : 0) * D];
            if (i0 + at < n) v += weight[at] * x;
        }
    }
    l = wave_sum(l);
#pragma unroll
    for (int x = 8; x < 64; x *= 2)
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j] += __shfl_xor(v[j], x);
    __syncthreads();
    if (lane == 0) parts[wave] = l;
    if (lane < 8) sums[wave][lane] = v;
    __syncthreads();
    if (threadIdx.x >= 8) return;
    store_joined(p, out * D + blockIdx.y * 32 + piece * 4, (sums[0][piece] + sums[1][piece]) + (sums[2][piece] + sums[3][piece]),
                 (parts[0] + parts[1]) + (parts[2] + parts[3]));
}

// How the rows and positions are cut: rows of a tile, and a chunk's positions, so many that there are about 1024 workgroups where every sequence fills its
// table, and 256 at least (two steps of each wave).  With 1024, 2048, 4096 and 8192: 64 sequences of 1000 to 8000 tokens 70, 72, 72 and 80 us, one of
// 131071 43, 45, 58 and 58; fewer were not tried (a CU has three at a time, with heads of 64 four).  A table has room for more than a sequence holds, and only the
// part that is held has work: 16 sequences of 8000, 32 heads of 128 on 8, take 33 us in a table for 8000 and 72 in one for 131072.
struct CachePlan {
    int32_t r, row_tiles;
    int64_t chunk, chunks, rows;
};
static int cache_plan(int64_t count, int64_t table_row, int64_t page, int64_t fresh, int64_t H, int64_t KV, CachePlan* c) {
    const int64_t room = table_row * page, rows = fresh * (H / KV);
    c->r = rows > 16 ? 2 : 1;
    const int64_t row_tiles = (rows + 16 * c->r - 1) / (16 * c->r), units = count * KV * row_tiles;
    if (room > (1 << 30) || units >= (1 << 23)) return LBA_ERR_SHAPE;
    c->row_tiles = (int32_t)row_tiles;
    c->chunk = (room * units + 1023) / 1024;
    if (c->chunk > room) c->chunk = room;                // (and within 32 bits)
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
    const bool fine = take_fine(&type);
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
    p.o_type = o_type; p.fine = fine || o_type == LBA_F32; p.part = (float*)workspace; p.room = (int32_t)(c.table_row * c.page);
    if (!lines) p.room = 0;                              // nothing is held anywhere
    p.chunk = (int32_t)plan.chunk; p.chunks = (int32_t)plan.chunks; p.row_tiles = plan.row_tiles;
    const hipStream_t st = (hipStream_t)hip_stream;
    if (type == LBA_F32) launch_cache_attn<float>(p, plan.r, st); else launch_cache_attn<bf16_t>(p, plan.r, st);
    if (plan.chunks > 1) {
        // a row's chunks one after another by one group of lanes, or side by side (64 sequences of up to 4 chunks, 2048 rows: 16 us side by side)
        const int per = 256 / (c.D / 4);
        if (plan.chunks <= 16) hipLaunchKernelGGL(cache_join_few_kernel, dim3((unsigned)((plan.rows + per - 1) / per)), dim3(256), 0, st, p, 16 * plan.r, plan.rows);
        else hipLaunchKernelGGL(cache_join_kernel, dim3((unsigned)plan.rows, (unsigned)c.D / 32), dim3(256), 0, st, p, 16 * plan.r);
    }
    return hipGetLastError() == hipSuccess ? LBA_OK : LBA_ERR_LAUNCH;
}

}  // extern "C"

// lba_cache_attn.hip -- attention of new tokens over a cache of 4 bits an element: one wave to a token's query head.
#include "lba_cache.h"

namespace lba {

struct CacheAttnParams {
    CacheParams c;
    const void* Q;
    void* O;
    CodeFmt fmt;
    lba_strides q;
    int32_t fresh, H, group;
    float scale;
};

__device__ __forceinline__ float cache_value(const CacheParams& c, const uint8_t* codes, const uint8_t* scales, int64_t line, int d) {
    return four_value(codes[line * (c.D / 2) + d / 2] >> (d % 2 * 4)) * power_of(scales[line * (c.D / 32) + d / 32]);
}

template <typename T, typename TO>
__global__ __launch_bounds__(64) void cache_attn_plain_kernel(CacheAttnParams p) {
    __shared__ float q[128], w[64];
    const int lane = threadIdx.x, D = p.c.D;
    const int64_t total = (int64_t)p.c.count * p.fresh * p.H;
    for (int64_t i = blockIdx.x; i < total; i += gridDim.x) {
        const int h = (int)(i % p.H), kv = h / p.group;
        const int64_t t = i / p.H;
        const int b = (int)(t / p.fresh);
        const int64_t seen = min((int64_t)p.c.lens[b] - p.fresh + t % p.fresh + 1, p.c.table_row * p.c.page);
        TO* o = (TO*)p.O + i * D;
        __syncthreads();
        for (int d = lane; d < D; d += 64) q[d] = load_one((const T*)p.Q + t * p.q.row + (int64_t)h * p.q.head + d);
        float m = -__builtin_inff(), l = 0.0f, acc0 = 0.0f, acc1 = 0.0f;
        for (int64_t j0 = 0; j0 < seen; j0 += 64) {
            __syncthreads();
            float s = -__builtin_inff();
            const int64_t mine = j0 + lane < seen ? line_of(p.c, b, j0 + lane, kv) : -1;
            if (mine >= 0) {
                s = 0.0f;
                for (int d = 0; d < D; ++d) s = fmaf(q[d], cache_value(p.c, p.c.k, p.c.k_scale, mine, d), s);
                s *= p.scale;
            }
            float top = s;
            for (int x = 32; x; x /= 2) top = fmaxf(top, __shfl_xor(top, x));
            top = fmaxf(top, m);
            const float base = top == -__builtin_inff() ? 0.0f : top;
            const float e = mine >= 0 ? exp_near(s - base) : 0.0f, f = exp_near(m - base);
            m = top;
            l = l * f + wave_sum(e);
            w[lane] = e;
            __syncthreads();
            acc0 *= f; acc1 *= f;
            const int n = (int)min((int64_t)64, seen - j0);
            for (int j = 0; j < n; ++j) {
                const int64_t line = line_of(p.c, b, j0 + j, kv);
                if (line < 0) continue;
                if (lane < D) acc0 = fmaf(w[j], cache_value(p.c, p.c.v, p.c.v_scale, line, lane), acc0);
                if (lane + 64 < D) acc1 = fmaf(w[j], cache_value(p.c, p.c.v, p.c.v_scale, line, lane + 64), acc1);
            }
        }
        const bool some = l > 0.0f || l != l;
        const float inv = some ? 1.0f / l : 0.0f;
        if (lane < D) store_one(o + lane, some ? acc0 * inv : 0.0f, p.fmt);
        if (lane + 64 < D) store_one(o + lane + 64, some ? acc1 * inv : 0.0f, p.fmt);
    }
}

}  // namespace lba

using namespace lba;

extern "C" {

size_t lba_cache_attention_workspace_bytes(int64_t count, int64_t table_row, int32_t page, int64_t fresh, int64_t H, int32_t KV, int32_t D) {
    (void)count; (void)table_row; (void)page; (void)fresh; (void)H; (void)KV; (void)D;
    return 0;
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
    const size_t need = lba_cache_attention_workspace_bytes(c.count, c.table_row, c.page, fresh, H, c.KV, c.D);
    if (need > 0) {
        if (!workspace) return LBA_ERR_NULL;
        if ((uintptr_t)workspace % 256 != 0) return LBA_ERR_ALIGN;
        if (workspace_bytes < need) return LBA_ERR_SHAPE;
    }
    p.Q = Q; p.O = O; p.q = q_at; p.fresh = (int32_t)fresh; p.H = (int32_t)H; p.group = (int32_t)(H / c.KV); p.scale = scale;
    if (o_type == LBA_CODE8) p.fmt = make_code_fmt(o_fmt);
    const int64_t rows = c.count * fresh * H;
    const dim3 grid((unsigned)(rows < (1 << 20) ? rows : (1 << 20)));
    const hipStream_t st = (hipStream_t)hip_stream;
#define LBA_CACHE_ATTN(T) \
    do { \
        if (o_type == LBA_F32) hipLaunchKernelGGL((cache_attn_plain_kernel<T, float>), grid, dim3(64), 0, st, p); \
        else if (o_type == LBA_BF16) hipLaunchKernelGGL((cache_attn_plain_kernel<T, bf16_t>), grid, dim3(64), 0, st, p); \
        else hipLaunchKernelGGL((cache_attn_plain_kernel<T, uint8_t>), grid, dim3(64), 0, st, p); \
    } while (0)
    if (type == LBA_F32) LBA_CACHE_ATTN(float); else LBA_CACHE_ATTN(bf16_t);
#undef LBA_CACHE_ATTN
    return hipGetLastError() == hipSuccess ? LBA_OK : LBA_ERR_LAUNCH;
}

}  // extern "C"

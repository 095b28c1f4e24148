// lba_cache.hip -- keys and values to and from a cache of 4 bits an element.
//
// A lane has eight consecutive elements, four lanes a block of 32: the block's largest size is the integer maximum of the elements' bits, which
// puts infinities and NaN above all numbers, its power of two comes from that number's exponent field, and codes are rounded by integer
// arithmetic on u = |x| / 2^e (exact: a power of two).  Bound by memory: elements in or out once, codes once.
#include "lba_cache.h"

namespace lba {

struct CacheRows {
    CacheParams c;
    const int32_t* starts;
    void *K, *V;
    lba_strides k, v;
    int32_t T, clear;
};

int cache_params(const lba_cache4& c, CacheParams* p) {
    if (c.pages < 0 || c.pages > 2147483647LL || c.table_row < 0 || c.table_row > 2147483647LL || c.count < 0 || c.count > (1 << 20)) return LBA_ERR_SHAPE;
    if (c.page < 1 || c.page > 65536 || c.KV < 0 || c.KV > 65535 || c.D < 32 || c.D > 128 || c.D % 32 != 0) return LBA_ERR_SHAPE;
    p->k = c.k; p->k_scale = c.k_scale; p->v = c.v; p->v_scale = c.v_scale; p->table = c.table; p->lens = c.lens;
    p->pages = c.pages; p->table_row = c.table_row; p->count = (int32_t)c.count; p->page = c.page; p->KV = c.KV; p->D = c.D;
    // floor(x / d) for x < 2^32: with 2^s the first power at or above d and m = floor(2^32 (2^s - d) / d) + 1,
    // (t + (x - t) / 2) / 2^(s - 1) where t is the high word of m x
    uint32_t s = 0;
    while ((1 << s) < c.page) ++s;
    p->page_shift = s;
    p->page_mul = (uint32_t)((((uint64_t)1 << 32) * (((uint64_t)1 << s) - (uint64_t)c.page)) / (uint64_t)c.page + 1);
    return LBA_OK;
}

// where row t's position is in head `head`: a line, -1: its sequence holds nothing there, -2: the row has no sequence
__device__ __forceinline__ int64_t row_line(const CacheRows& p, int t, int head) {
    const int b = sequence_of(p.starts, p.T, p.c.count, t);
    if (b < 0) return -2;
    const Rows r = rows_of(p.starts, p.T, p.c.count, b);
    return line_of(p.c, b, (int64_t)p.c.lens[b] - r.n + (t - r.first), head);
}

__device__ __forceinline__ uint32_t four_code(float x, float inverse) {
    const float u = fabsf(x) * inverse;
    const uint32_t b = __float_as_uint(u);
    // from 1 on one mantissa bit is kept; below, steps of 0.5 are what a number of 2^22 has
    uint32_t c = ((b + 0x1FFFFFu + ((b >> 22) & 1u)) >> 22) - 252u;
    if (u < 1.0f) c = __float_as_uint(u + 4194304.0f) - __float_as_uint(4194304.0f);
    return min(c, 7u) | ((__float_as_uint(x) >> 28) & 8u);
}

template <typename T> __global__ __launch_bounds__(256) void cache_write_kernel(CacheRows p) {
    const int parts = p.c.D / 8;
    const int64_t total = (int64_t)p.T * p.c.KV * parts;
    const T* X = (const T*)(blockIdx.y ? p.V : p.K);
    const lba_strides at = blockIdx.y ? p.v : p.k;
    uint8_t* codes = blockIdx.y ? p.c.v : p.c.k;
    uint8_t* scales = blockIdx.y ? p.c.v_scale : p.c.k_scale;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < total; i += (int64_t)gridDim.x * 256) {    // whole groups of four lanes
        const int part = (int)(i % parts), head = (int)(i / parts % p.c.KV), t = (int)(i / parts / p.c.KV);
        const int64_t line = row_line(p, t, head);
        float x[8];
        load_vec<8>(X + (int64_t)t * at.row + (int64_t)head * at.head + part * 8, x);
        uint32_t top = 0;
#pragma unroll
        for (int j = 0; j < 8; ++j) top = max(top, __float_as_uint(x[j]) & 0x7FFFFFFFu);
        top = max(top, (uint32_t)__shfl_xor((int)top, 1));
        top = max(top, (uint32_t)__shfl_xor((int)top, 2));
        int e = (int)(top >> 23) - 127 - 2 + ((top & 0x7FFFFFu) > 0x400000u ? 1 : 0);
        e = min(max(e, -100), 125);
        const float inverse = __uint_as_float((uint32_t)(127 - e) << 23);
        uint32_t w = 0;
#pragma unroll
        for (int j = 0; j < 8; ++j) w |= four_code(x[j], inverse) << (4 * j);
        const bool broken = top >= 0x7F800000u;
        if (line < 0) continue;
        typedef uint32_t word __attribute__((aligned(1)));
        *(word*)(codes + line * (p.c.D / 2) + part * 4) = broken ? 0u : w;
        if (part % 4 == 0) scales[line * (p.c.D / 32) + part / 4] = broken ? 255 : (uint8_t)(e + 127);
    }
}

template <typename T> __global__ __launch_bounds__(256) void cache_read_kernel(CacheRows p) {
    const int parts = p.c.D / 8;
    const int64_t total = (int64_t)p.T * p.c.KV * parts;
    T* X = (T*)(blockIdx.y ? p.V : p.K);
    const lba_strides at = blockIdx.y ? p.v : p.k;
    const uint8_t* codes = blockIdx.y ? p.c.v : p.c.k;
    const uint8_t* scales = blockIdx.y ? p.c.v_scale : p.c.k_scale;
    const CodeFmt none = {};
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < total; i += (int64_t)gridDim.x * 256) {
        const int part = (int)(i % parts), head = (int)(i / parts % p.c.KV), t = (int)(i / parts / p.c.KV);
        const int64_t line = row_line(p, t, head);
        if (line == -2 && !p.clear) continue;
        float x[8] = {0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f};
        if (line >= 0) {
            typedef uint32_t word __attribute__((aligned(1)));
            const uint32_t w = *(const word*)(codes + line * (p.c.D / 2) + part * 4);
            const float s = power_of(scales[line * (p.c.D / 32) + part / 4]);
#pragma unroll
            for (int j = 0; j < 8; ++j) x[j] = four_value(w >> (4 * j)) * s;
        }
        store_vec<8>(X + (int64_t)t * at.row + (int64_t)head * at.head + part * 8, x, none);
    }
}

static int cache_rows(const lba_cache4& c, const int32_t* starts, int64_t T, const void* K, lba_strides k_at, const void* V, lba_strides v_at, int32_t type,
                      CacheRows* p) {
    int rc = cache_params(c, &p->c);
    if (rc == LBA_OK) rc = check_heads(T, c.KV, c.D);
    if (rc == LBA_OK) rc = check_strides(k_at);
    if (rc == LBA_OK) rc = check_strides(v_at);
    if (rc == LBA_OK && !starts && (c.count < 1 ? T != 0 : T % c.count != 0)) rc = LBA_ERR_SHAPE;
    if (rc == LBA_OK) rc = check_float_type(type);
    if (rc != LBA_OK) return rc;
    p->starts = starts; p->K = (void*)K; p->V = (void*)V; p->k = k_at; p->v = v_at; p->T = (int32_t)T;
    if (T == 0 || c.KV == 0) return LBA_OK;
    const bool table = c.count > 0 && c.table_row > 0, lines = table && c.pages > 0;
    if (!K || !V || (c.count > 0 && !c.lens) || (table && !c.table) || (lines && (!c.k || !c.k_scale || !c.v || !c.v_scale))) return LBA_ERR_NULL;
    return LBA_OK;
}

static dim3 cache_grid(const CacheRows& p) {
    const int64_t blocks = ((int64_t)p.T * p.c.KV * (p.c.D / 8) + 255) / 256;
    return dim3((unsigned)(blocks < (1 << 20) ? blocks : (1 << 20)), 2);
}

}  // namespace lba

using namespace lba;

extern "C" {

int lba_cache_write(lba_cache4 c, const int32_t* starts, int64_t T, const void* K, lba_strides k_at, const void* V, lba_strides v_at, int32_t type,
                    void* hip_stream) {
    CacheRows p = {};
    const int rc = cache_rows(c, starts, T, K, k_at, V, v_at, type, &p);
    if (rc != LBA_OK || p.T == 0 || p.c.KV == 0 || p.c.count == 0) return rc;
    if (type == LBA_F32) hipLaunchKernelGGL((cache_write_kernel<float>), cache_grid(p), dim3(256), 0, (hipStream_t)hip_stream, p);
    else hipLaunchKernelGGL((cache_write_kernel<bf16_t>), cache_grid(p), dim3(256), 0, (hipStream_t)hip_stream, p);
    return hipGetLastError() == hipSuccess ? LBA_OK : LBA_ERR_LAUNCH;
}

int lba_cache_read(lba_cache4 c, const int32_t* starts, int64_t T, void* K, lba_strides k_at, void* V, lba_strides v_at, int32_t type, int32_t clear,
                   void* hip_stream) {
    CacheRows p = {};
    const int rc = cache_rows(c, starts, T, K, k_at, V, v_at, type, &p);
    if (rc != LBA_OK || p.T == 0 || p.c.KV == 0 || (p.c.count == 0 && !clear)) return rc;
    p.clear = clear != 0;
    if (type == LBA_F32) hipLaunchKernelGGL((cache_read_kernel<float>), cache_grid(p), dim3(256), 0, (hipStream_t)hip_stream, p);
    else hipLaunchKernelGGL((cache_read_kernel<bf16_t>), cache_grid(p), dim3(256), 0, (hipStream_t)hip_stream, p);
    return hipGetLastError() == hipSuccess ? LBA_OK : LBA_ERR_LAUNCH;
}

}  // extern "C"

// lba_cache.hip -- keys and values to and from a cache of 4 bits an element.
//
// A workgroup finds its rows' places first, a lane a row, and then takes their heads' keys and values together.  A lane has eight consecutive
// elements, four lanes a block of 32: the block's largest size is the integer maximum of the elements' bits, which puts infinities and NaN
// above all numbers, and its power of two comes from that number's exponent field; the conversion to codes divides by it and rounds to
// nearest even.  Bound by memory: elements in or out once, codes once.
#include "lba_cache.h"

namespace lba {

struct CacheRows {
    CacheParams c;
    const int32_t* starts;
    void *K, *V;
    lba_strides k, v;
    int32_t T, clear, rows;  // rows of a workgroup
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

constexpr int kCacheRows = 8;                            // rows of a workgroup at most

// where row t's position is in head 0: a line, -1: its sequence holds nothing there, -2: the row has no sequence
__device__ __forceinline__ int64_t row_line(const CacheRows& p, int t) {
    const int b = sequence_of(p.starts, p.T, p.c.count, t);
    if (b < 0) return -2;
    const Rows r = rows_of(p.starts, p.T, p.c.count, b);
    return line_of(p.c, b, (int64_t)p.c.lens[b] - r.n + (t - r.first), 0);
}

// f(row of the tensor, line of its head (or -1, -2 as above), head, which eight elements, 0: keys, 1: values): for all of the workgroup's rows.  Four
// neighbouring lanes have a block of 32 elements or nothing.
template <typename F> __device__ __forceinline__ void for_rows(const CacheRows& p, F f) {
    __shared__ int64_t lines[kCacheRows];
    const int parts = p.c.D / 8, items = p.c.KV * parts;
    for (int64_t t0 = (int64_t)blockIdx.x * p.rows; t0 < p.T; t0 += (int64_t)gridDim.x * p.rows) {
        const int rows = (int)min((int64_t)p.rows, p.T - t0);
        __syncthreads();
        if ((int)threadIdx.x < rows) lines[threadIdx.x] = row_line(p, (int)t0 + threadIdx.x);
        __syncthreads();
        for (int i = threadIdx.x; i < 2 * rows * items; i += 256) {
            const int head = i / parts % p.c.KV, x = i / items;
            const int64_t line = lines[x >> 1];
            f(t0 + (x >> 1), line < 0 ? line : line + (int64_t)head * p.c.page, head, i % parts, x & 1);
        }
    }
}

typedef uint32_t any_word __attribute__((aligned(1)));

template <typename T> __global__ __launch_bounds__(256) void cache_write_kernel(CacheRows p) {
    for_rows(p, [&](int64_t t, int64_t line, int head, int part, int values) {
        const lba_strides at = values ? p.v : p.k;
        float x[8];
        load_vec<8>((const T*)(values ? p.V : p.K) + t * at.row + (int64_t)head * at.head + part * 8, x);
        uint32_t top = 0;
#pragma unroll
        for (int j = 0; j < 8; ++j) top = max(top, __float_as_uint(x[j]) & 0x7FFFFFFFu);
        top = max(top, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)top, 0xB1, 0xF, 0xF, true));                    // lanes 1 and 2 apart, of four
        top = max(top, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)top, 0x4E, 0xF, 0xF, true));
        int e = (int)(top >> 23) - 127 - 2 + ((top & 0x7FFFFFu) > 0x400000u ? 1 : 0);
        e = min(max(e, -100), 125);
        const float power = __uint_as_float((uint32_t)(127 + e) << 23);
        uint32_t w = 0;
        w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[0], x[1], power, 0);
        w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[2], x[3], power, 1);
        w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[4], x[5], power, 2);
        w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[6], x[7], power, 3);
        const bool broken = top >= 0x7F800000u;
        if (line < 0) return;
        *(any_word*)((values ? p.c.v : p.c.k) + line * (p.c.D / 2) + part * 4) = broken ? 0u : w;
        if (part % 4 == 0) (values ? p.c.v_scale : p.c.k_scale)[line * (p.c.D / 32) + part / 4] = broken ? 255 : (uint8_t)(e + 127);
    });
}

template <typename T> __global__ __launch_bounds__(256) void cache_read_kernel(CacheRows p) {
    const CodeFmt none = {};
    for_rows(p, [&](int64_t t, int64_t line, int head, int part, int values) {
        if (line == -2 && !p.clear) return;
        const lba_strides at = values ? p.v : p.k;
        float x[8] = {0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f};
        if (line >= 0) {
            const uint32_t w = *(const any_word*)((values ? p.c.v : p.c.k) + line * (p.c.D / 2) + part * 4);
            const float s = power_of((values ? p.c.v_scale : p.c.k_scale)[line * (p.c.D / 32) + part / 4]);
#pragma unroll
            for (int j = 0; j < 8; ++j) x[j] = four_value(w >> (4 * j)) * s;
        }
        store_vec<8>((T*)(values ? p.V : p.K) + t * at.row + (int64_t)head * at.head + part * 8, x, none);
    });
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

// Eight rows of a workgroup where that leaves two workgroups a CU, one where there are few.
static dim3 cache_grid(CacheRows* p) {
    p->rows = p->T / 512 < 1 ? 1 : p->T / 512 < kCacheRows ? p->T / 512 : kCacheRows;
    const int64_t blocks = ((int64_t)p->T + p->rows - 1) / p->rows;
    return dim3((unsigned)(blocks < (1 << 20) ? blocks : (1 << 20)));
}

}  // namespace lba

using namespace lba;

extern "C" {

int lba_cache_write(lba_cache4 c, const int32_t* starts, int64_t T, const void* K, lba_strides k_at, const void* V, lba_strides v_at, int32_t type,
                    void* hip_stream) {
    CacheRows p = {};
    const int rc = cache_rows(c, starts, T, K, k_at, V, v_at, type, &p);
    if (rc != LBA_OK || p.T == 0 || p.c.KV == 0 || p.c.count == 0) return rc;
    if (type == LBA_F32) hipLaunchKernelGGL((cache_write_kernel<float>), cache_grid(&p), dim3(256), 0, (hipStream_t)hip_stream, p);
    else hipLaunchKernelGGL((cache_write_kernel<bf16_t>), cache_grid(&p), dim3(256), 0, (hipStream_t)hip_stream, p);
    return hipGetLastError() == hipSuccess ? LBA_OK : LBA_ERR_LAUNCH;
}

int lba_cache_read(lba_cache4 c, const int32_t* starts, int64_t T, void* K, lba_strides k_at, void* V, lba_strides v_at, int32_t type, int32_t clear,
                   void* hip_stream) {
    CacheRows p = {};
    const int rc = cache_rows(c, starts, T, K, k_at, V, v_at, type, &p);
    if (rc != LBA_OK || p.T == 0 || p.c.KV == 0 || (p.c.count == 0 && !clear)) return rc;
    p.clear = clear != 0;
    if (type == LBA_F32) hipLaunchKernelGGL((cache_read_kernel<float>), cache_grid(&p), dim3(256), 0, (hipStream_t)hip_stream, p);
    else hipLaunchKernelGGL((cache_read_kernel<bf16_t>), cache_grid(&p), dim3(256), 0, (hipStream_t)hip_stream, p);
    return hipGetLastError() == hipSuccess ? LBA_OK : LBA_ERR_LAUNCH;
}

}  // extern "C"

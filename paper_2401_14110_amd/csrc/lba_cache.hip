// lba_cache.hip -- keys and values to and from a cache of 4 bits an element.
//
// A workgroup finds its rows' places, a lane a row, and takes their heads' keys and values together.  A lane has eight consecutive elements,
// four lanes a block of 32: the block's largest size is the integer maximum of the elements' bits, which puts infinities and NaN above all
// numbers, and its power of two comes from that number's exponent field; the conversion to codes divides by it and rounds to nearest even.
// Bound by memory: elements in or out once, codes once.  All workgroups run at the same time, so that a launch takes as long as one's chain of reads
// and the instructions of all: a lane's place in a head is worked out once, not per row (11118 tokens, 8 heads of 128, 58 MB each way: 17 and
// 21 us with divisions for every eight elements, 13.5 and 13.4 so, 11 at a copy's rate).
#include "lba_cache.h"

namespace lba {

struct CacheRows {
    CacheParams c;
    const int32_t* starts;
    void *K, *V;
    lba_strides k, v;
    int32_t T, clear, rows;  // rows of a workgroup
    int32_t parts, items;    // groups of eight elements of a head, and of all heads
    Divisor by_parts, by_items;
};

int cache_params(const lba_cache4& c, CacheParams* p) {
    if (c.pages < 0 || c.pages > 2147483647LL || c.table_row < 0 || c.table_row > 2147483647LL || c.count < 0 || c.count > (1 << 20)) return LBA_ERR_SHAPE;
    if (c.page < 1 || c.page > 65536 || c.KV < 0 || c.KV > 65535 || c.D < 32 || c.D > 128 || c.D % 32 != 0) return LBA_ERR_SHAPE;
    p->k = c.k; p->k_scale = c.k_scale; p->v = c.v; p->v_scale = c.v_scale; p->table = c.table; p->lens = c.lens;
    p->pages = c.pages; p->table_row = c.table_row; p->count = (int32_t)c.count; p->page = c.page; p->KV = c.KV; p->D = c.D;
    p->by_page = divisor((uint32_t)c.page);
    return LBA_OK;
}

constexpr int kCacheRows = 8;                            // rows of a workgroup at most

// where row t's position has its codes of head 0, in bytes: -1: its sequence holds nothing there, -2: the row has no sequence
__device__ __forceinline__ int64_t row_codes(const CacheRows& p, int t) {
    const int b = sequence_of(p.starts, p.T, p.c.count, t);
    if (b < 0) return -2;
    const Rows r = rows_of(p.starts, p.T, p.c.count, b);
    const int64_t line = line_of(p.c, b, (int64_t)p.c.lens[b] - r.n + (t - r.first), 0);
    return line < 0 ? line : line * (p.c.D / 2);
}

// All elements of the workgroup's rows: a lane has eight of one head (four neighbouring lanes a block of 32) and goes over rows, kCacheBatch at a time and
// their keys and values together, so that what a row costs is a few additions.  begin(n, keys, values, codes) starts what the n-th row of the batch needs
// from memory and end(..) ends it: where the eight elements are in the tensors, where their codes are (-1, -2 as above).  EARLY: begin does
// not look at the codes, and is called while their places are looked up.
constexpr int kCacheBatch = 2;
template <bool EARLY, typename Begin, typename End> __device__ __forceinline__ void for_rows(const CacheRows& p, Begin begin, End end) {
    __shared__ int64_t places[kCacheRows];
    const int per = max(1, 256 / p.items);               // rows at once
    const int g = p.by_items.of(threadIdx.x), start = threadIdx.x - g * p.items;     // (more than 256 lanes' worth of heads: g is 0)
    for (int64_t t0 = (int64_t)blockIdx.x * p.rows; t0 < p.T; t0 += (int64_t)gridDim.x * p.rows) {
        const int rows = (int)min((int64_t)p.rows, p.T - t0);
        auto batch = [&](int in, int x0, bool placed, auto f) {
            const int head = p.by_parts.of(in), part = in - head * p.parts;
            const int64_t k = (t0 + x0) * p.k.row + (int64_t)head * p.k.head + part * 8, v = (t0 + x0) * p.v.row + (int64_t)head * p.v.head + part * 8;
            const int64_t codes = (int64_t)head * p.c.page * (p.c.D / 2) + part * 4;
#pragma unroll
            for (int n = 0; n < kCacheBatch; ++n)
                if (x0 + n * per < rows) {
                    const int64_t place = placed ? places[x0 + n * per] : -1;
                    f(n, k + (int64_t)(n * per) * p.k.row, v + (int64_t)(n * per) * p.v.row, place < 0 ? place : place + codes);
                }
        };
        bool begun = EARLY && g < per;
        __syncthreads();                                 // the rows before are done
        if (begun) batch(start, g, false, begin);
        if ((int)threadIdx.x < rows) places[threadIdx.x] = row_codes(p, (int)t0 + threadIdx.x);
        __syncthreads();
        if (g >= per) continue;
        for (int in = start; in < p.items; in += 256)
            for (int x0 = g; x0 < rows; x0 += per * kCacheBatch) {
                if (!begun) batch(in, x0, true, begin);
                begun = false;
                batch(in, x0, true, end);
            }
    }
}

typedef uint32_t any_word __attribute__((aligned(1)));

// eight elements to their codes, and the block's power
template <typename B> __device__ __forceinline__ void eight_to_codes(const Raw<B, 8>& r, uint8_t* to, uint8_t* scales, int64_t at) {
    float x[8];
    uint32_t top = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        x[j] = raw_at<8>(r, j);
        top = max(top, __float_as_uint(x[j]) & 0x7FFFFFFFu);
    }
    top = max(top, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)top, 0xB1, 0xF, 0xF, true));                        // lanes 1 and 2 apart, of four
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
    if (at < 0) return;
    *(any_word*)(to + at) = broken ? 0u : w;
    if ((at & 15) == 0) scales[at >> 4] = broken ? 255 : (uint8_t)(e + 127);           // a block has 16 bytes of codes
}

template <typename T> __global__ __launch_bounds__(256, sizeof(T) == 2 ? 6 : 4) void cache_write_kernel(CacheRows p) {
    typedef typename Bits<T>::type B;
    Raw<B, 8> keys[kCacheBatch], values[kCacheBatch];
    for_rows<true>(p, [&](int n, int64_t k, int64_t v, int64_t) {
        keys[n] = load_raw<B, 8>((const B*)p.K + k, 8);
        values[n] = load_raw<B, 8>((const B*)p.V + v, 8);
    }, [&](int n, int64_t, int64_t, int64_t codes) {
        eight_to_codes<B>(keys[n], p.c.k, p.c.k_scale, codes);
        eight_to_codes<B>(values[n], p.c.v, p.c.v_scale, codes);
    });
}

template <typename T> __global__ __launch_bounds__(256) void cache_read_kernel(CacheRows p) {
    const CodeFmt none = {};
    uint32_t keys[kCacheBatch], values[kCacheBatch];
    uint8_t key_power[kCacheBatch], value_power[kCacheBatch];
    auto store = [&](void* to, uint32_t codes, uint32_t power) {
        const float s = __uint_as_float(power << 23);    // (the conversion reads an exponent of all ones as NaN)
        const uint32_t w = power == 0 ? 0u : codes;
        typedef __bf16 two __attribute__((ext_vector_type(2)));
        const two y[4] = {__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, 0), __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, 1),
                          __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, 2), __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, 3)};
        float x[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) x[j] = (float)y[j / 2][j % 2];
        store_vec<8>((T*)to, x, none);
    };
    for_rows<false>(p, [&](int n, int64_t, int64_t, int64_t codes) {
        keys[n] = values[n] = 0;
        key_power[n] = value_power[n] = 0;
        if (codes < 0) return;
        keys[n] = *(const any_word*)(p.c.k + codes);
        values[n] = *(const any_word*)(p.c.v + codes);
        key_power[n] = p.c.k_scale[codes >> 4];
        value_power[n] = p.c.v_scale[codes >> 4];
    }, [&](int n, int64_t k, int64_t v, int64_t codes) {
        if (codes == -2 && !p.clear) return;
        store((T*)p.K + k, keys[n], key_power[n]);
        store((T*)p.V + v, values[n], value_power[n]);
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
    p->parts = c.D / 8; p->items = c.KV * p->parts;
    p->by_parts = divisor(p->parts); p->by_items = divisor(p->items > 0 ? p->items : 1);
    if (T == 0 || c.KV == 0) return LBA_OK;
    const bool table = c.count > 0 && c.table_row > 0, lines = table && c.pages > 0;
    if (!K || !V || (c.count > 0 && !c.lens) || (table && !c.table) || (lines && (!c.k || !c.k_scale || !c.v || !c.v_scale))) return LBA_ERR_NULL;
    return LBA_OK;
}

// Eight rows of a workgroup where that leaves two workgroups a CU, one where there are few.  (11118 tokens: 1, 2 and 4 rows 28, 21 and 18 us when eight
// took 17; now 16 take 14.3 and 13 where eight take 13.6 and 13.4.)
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

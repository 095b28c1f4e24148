// lba_cache.h -- the cache of 4 bits an element on the device: where a position is, what a code stands for.
#ifndef LBA_CACHE_H_
#define LBA_CACHE_H_

#include "lba_attn_device.h"

namespace lba {

// x / d without a division, for any x below 2^32 and d from 1 to 2^31: with 2^s the first power at or above d and m = floor(2^32 (2^s - d) / d) + 1,
// (t + (x - t) / 2) / 2^(s - 1) where t is the high word of m x
struct Divisor {
    uint32_t mul, shift;

    __device__ __forceinline__ uint32_t of(uint32_t x) const {
        const uint32_t t = __umulhi(mul, x);
        return shift == 0 ? x : (t + ((x - t) >> 1)) >> (shift - 1);
    }
};
inline Divisor divisor(uint32_t d) {
    uint32_t s = 0;
    while (((uint64_t)1 << s) < d) ++s;
    return {(uint32_t)((((uint64_t)1 << 32) * (((uint64_t)1 << s) - d)) / d + 1), s};
}

struct CacheParams {
    uint8_t *k, *k_scale, *v, *v_scale;
    const int32_t *table, *lens;
    int64_t pages, table_row;
    int32_t count, page, KV, D;
    Divisor by_page;

    __device__ __forceinline__ int64_t page_div(int64_t at) const { return by_page.of((uint32_t)at); }               // (positions are below 2^31)
    __device__ __forceinline__ int32_t page_mod(int64_t at) const { return (int32_t)(at - page_div(at) * page); }
};

int cache_params(const lba_cache4& c, CacheParams* p);

// The line of a head's pages that sequence b's position `at` has, counted over the whole cache, -1: none.
__device__ __forceinline__ int64_t line_of(const CacheParams& p, int b, int64_t at, int head) {
    if (at < 0) return -1;
    const int64_t column = p.page_div(at);
    if (column >= p.table_row) return -1;
    const int64_t page = p.table[(int64_t)b * p.table_row + column];
    if (page < 0 || page >= p.pages) return -1;
    return (page * p.KV + head) * p.page + p.page_mod(at);
}

}  // namespace lba
#endif

// lba_cache_attn.h -- parameters of attention over the cache
#ifndef LBA_CACHE_ATTN_H_
#define LBA_CACHE_ATTN_H_

#include "lba_cache.h"

namespace lba {

typedef float f32x4_c __attribute__((ext_vector_type(4)));

struct CacheAttnParams {
    CacheParams c;
    const void* Q;
    void* O;
    float* part;             // [rows][chunks][D]: sums; then [rows][chunks][2]: maximum, sum of weights; null: one chunk
    CodeFmt fmt;
    lba_strides q;
    int32_t room;            // positions of a sequence's table
    int32_t fresh, H, group, o_type;
    int32_t fine;            // weights of bfloat16 queries are three pieces
    int32_t chunk, chunks, row_tiles;
    float scale;
};

// how many positions a row sees; of a tile its last row sees most
__device__ __forceinline__ int row_seen(const CacheAttnParams& p, int b, int row) {
    return (int)max((int64_t)0, min((int64_t)p.c.lens[b] - p.fresh + row / p.group + 1, (int64_t)p.room));
}

// the kernels of a type, with tiles of 16 r rows
template <typename T> void launch_cache_attn(const CacheAttnParams& p, int r, hipStream_t st);

}  // namespace lba
#endif

// lba_cache_attn_f32.hip -- attention over the cache with float32 queries
#include "lba_cache_attn_fwd.h"

namespace lba {
template void launch_cache_attn<float>(const CacheAttnParams& p, int r, hipStream_t st);
}

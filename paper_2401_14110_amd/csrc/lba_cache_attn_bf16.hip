// lba_cache_attn_bf16.hip -- attention over the cache with bfloat16 queries
#include "lba_cache_attn_fwd.h"

namespace lba {
template void launch_cache_attn<bf16_t>(const CacheAttnParams& p, int r, hipStream_t st);
}

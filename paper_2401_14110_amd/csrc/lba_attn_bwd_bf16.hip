// lba_attn_bwd_bf16.hip -- the gradients of attention on bfloat16
#include "lba_attn_bwd.h"

namespace lba {
template void launch_attn_dq<bf16_t>(const AttnParams& p, bool direct, hipStream_t st);
template void launch_attn_dkv<bf16_t>(const AttnParams& p, bool direct, hipStream_t st);
}

// lba_attn_bf16.hip -- attention on bfloat16
#include "lba_attn_fwd.h"

namespace lba {
template void launch_attn<bf16_t>(const AttnParams& p, bool direct, hipStream_t st);
}

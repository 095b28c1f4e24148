// lba_attn_bwd_f32.hip -- the gradients of attention on float32
#include "lba_attn_bwd.h"

namespace lba {
template void launch_attn_dq<float>(const AttnParams& p, bool direct, hipStream_t st);
template void launch_attn_dkv<float>(const AttnParams& p, bool direct, hipStream_t st);
}

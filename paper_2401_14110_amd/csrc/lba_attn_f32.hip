// lba_attn_f32.hip -- attention on float32
#include "lba_attn_fwd.h"

namespace lba {
template void launch_attn<float>(const AttnParams& p, bool direct, hipStream_t st);
}

// Instantiations of the dense tile for bfloat16 rows: codes of five exponent bits, which are laid out as bfloat16 numbers, and the gradient
// products.
#include "lba_dense.h"

namespace lba {
int launch_dense_bf16(const GemmParams& a, const GemmParams* b, const Beside* side, int tile, bool gated, int epi, hipStream_t st) {
    return launch_dense<ELEM_BF16>(a, b, side, tile, gated, epi, st);
}
}  // namespace lba

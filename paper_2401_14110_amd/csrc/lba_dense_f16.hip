// Instantiations of the dense tile for codes of two to four exponent bits.
#include "lba_dense.h"

namespace lba {
int launch_dense_f16(const GemmParams& a, const GemmParams* b, const Beside* side, int tile, bool gated, int epi, hipStream_t st) {
    return launch_dense<ELEM_F16>(a, b, side, tile, gated, epi, st);
}
}  // namespace lba

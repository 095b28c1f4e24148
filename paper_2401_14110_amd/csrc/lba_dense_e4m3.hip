// Instantiations of the dense tile for E4M3 codes.
#include "lba_dense.h"

namespace lba {
int launch_dense_e4m3(const GemmParams& a, const GemmParams* b, const Beside* side, int tile, bool gated, int epi, hipStream_t st) {
    return launch_dense<ELEM_E4M3>(a, b, side, tile, gated, epi, st);
}
}  // namespace lba

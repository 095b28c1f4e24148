// What the entry points of the dense product launch, without a GPU: lba_dense.hip as it is, and in place of the kernels' launchers ones that
// keep the products, the tile and the workgroups beside them.  tests/test_dense_launches_cpu.py builds and loads it.
#include "lba_dense.h"

namespace {
struct Record { int32_t tile, products; int64_t tiles, beside; };
Record seen[2];
int calls = 0;
int keep(const lba::GemmParams& a, const lba::GemmParams* b, const lba::Beside* side, int tile, bool gated, int epi) {
    lba::GemmParams x = a, y = b ? *b : a;
    const lba::TileShape s = lba::tile_shape(tile);
    const int64_t first = lba::dense_grid(x, s, gated), second = b ? lba::dense_grid(y, s, gated) : 0;
    const int64_t beside = !side ? 0 : epi == lba::EPI_BACKWARD ? (int64_t)side->job_blocks : (side->sums.cols + 15) / 16;
    if (calls < 2) seen[calls] = {tile, b ? 2 : 1, first + second, beside};
    ++calls;
    return LBA_OK;
}
}  // namespace

namespace lba {
#define LBA_KEEP(NAME) \
    int NAME(const GemmParams& a, const GemmParams* b, const Beside* side, int tile, bool gated, int epi, hipStream_t) { return keep(a, b, side, tile, gated, epi); }
LBA_KEEP(launch_dense_e4m3) LBA_KEEP(launch_dense_f16) LBA_KEEP(launch_dense_bf16)
void launch_dense_token(const TokenParams&, int, bool, hipStream_t) { ++calls; }
}  // namespace lba

extern "C" int take_launches(Record* out) {
    out[0] = seen[0];
    out[1] = seen[1];
    const int n = calls;
    calls = 0;
    return n;
}

// lba_attn.h -- parameters of the attention kernels
#ifndef LBA_ATTN_H_
#define LBA_ATTN_H_

#include "lba_attn_device.h"

namespace lba {

struct AttnParams {
    const void *Q, *K, *V;
    void* O;
    float* lse;
    CodeFmt fmt;
    // backward
    const void* G;
    void *dQ, *dK, *dV;
    float* delta;            // [T, H]: rowsum(G * O)
    const int32_t *starts, *starts_k;
    lba_strides q, k, v, dq, dk, dv;
    int32_t T, Tk, count, H, KV, group, D;
    int32_t causal, clear, o_type;
    int32_t fine;            // bfloat16 inputs: forward, weights are three pieces; backward, all tiles make rowsum(G * O) from the weights
    int32_t tiles, units;    // tiles of queries (keys) that there may be, and those of all heads
    int32_t slices;          // parts that a workgroup's steps are cut into, where there are few workgroups
    float* part;             // their sums: [slices][rows][D], behind them what else a row has
    float scale;
};

int attn_params(const lba_attn& a, AttnParams* p);       // checks and copies the description

constexpr int kTileRows = 128;                           // queries (keys, where keys have the sums) of a workgroup
constexpr int kClearBlocks = 16;                         // workgroups behind the others, for rows of no sequence
constexpr int64_t kMostUnits = 1 << 23;                  // workgroups of a launch: fewer than 2^32 lanes
constexpr int kMostSlices = 16;

// Whether rows can go to LDS in pieces of 16 aligned bytes (one more head or row keeps the place in a piece), 64 rows within 2^31 bytes.
inline bool whole_pieces(const void* x, const lba_strides& at, int64_t D, int64_t size) {
    return ((uintptr_t)x | (uintptr_t)(at.row * size) | (uintptr_t)(at.head * size) | (uintptr_t)(D * size)) % 16 == 0 && at.row < (1 << 22);
}

// How the three passes are cut: see attn_plan.
struct AttnPlan {
    int64_t tiles_q, tiles_k;            // that there may be
    int32_t slices, slices_dq, slices_dkv;
};
int attn_plan(const lba_attn& a, AttnPlan* plan);

template <typename T> void launch_attn_dq(const AttnParams& p, bool direct, hipStream_t st);
template <typename T> void launch_attn_dkv(const AttnParams& p, bool direct, hipStream_t st);
template <typename T> void launch_attn(const AttnParams& p, bool direct, hipStream_t st);

}  // namespace lba
#endif

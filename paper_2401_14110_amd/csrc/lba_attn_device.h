// lba_attn_device.h -- what the operators of lba_attention.h share: tensors of heads, packed sequences, refusals.
#ifndef LBA_ATTN_DEVICE_H_
#define LBA_ATTN_DEVICE_H_

#include "lba_attention.h"
#include "lba_layer_device.h"

namespace lba {

// rows first .. first + n - 1 of a tensor belong to a sequence
struct Rows {
    int first, n;
};

// Sequence b of `count` in a list of starts over T rows (null: equal lengths), kept inside the tensor whatever the list holds.
__device__ __forceinline__ Rows rows_of(const int32_t* starts, int T, int count, int b) {
    if (!starts) {
        const int n = T / count;
        return {b * n, n};
    }
    const int lo = min(max(starts[b], 0), T), hi = min(max(starts[b + 1], lo), T);
    return {lo, hi - lo};
}

// The sequence that row `t` belongs to, -1: none.  The last one whose start is not behind t (empty ones share their start with the next).
__device__ __forceinline__ int sequence_of(const int32_t* starts, int T, int count, int t) {
    if (count < 1) return -1;
    if (!starts) return t / (T / count);
    int lo = 0, hi = count;                              // starts[lo] <= t < starts[hi], were the list extended so
    while (hi - lo > 1) {
        const int mid = (lo + hi) / 2;
        if (starts[mid] <= t) lo = mid; else hi = mid;
    }
    const Rows r = rows_of(starts, T, count, lo);
    return t >= r.first && t < r.first + r.n ? lo : -1;
}

// ---- host checks ----------------------------------------------------------------------------

// whether LBA_FINE was in a type, which is without it then
inline bool take_fine(int32_t* type) {
    const bool fine = (*type & LBA_FINE) != 0;
    *type &= ~LBA_FINE;
    return fine;
}
inline int check_strides(const lba_strides& s) { return s.row < 0 || s.head < 0 ? LBA_ERR_SHAPE : LBA_OK; }
inline int check_heads(int64_t T, int64_t H, int64_t D) {
    return T < 0 || T > 2147483647LL || H < 0 || H > 65535 || D < 0 || D > 1024 ? LBA_ERR_SHAPE : LBA_OK;
}

}  // namespace lba
#endif

// lba_dense_index.h -- where the dense product's epilogue reads and writes.  Plain C++: tests/dense_index.cpp compares every element of a
// wave's part with 64-bit arithmetic.
#ifndef LBA_DENSE_INDEX_H_
#define LBA_DENSE_INDEX_H_

#include "lba_piece_index.h"

namespace lba {

// An element's index in two parts: `u` is the same for a wave in the tile (a scalar register), `o` a lane's 32-bit offset from it.
struct At { int64_t u; uint32_t o; };
template <typename T> LBA_HOST_DEVICE T* at(const T* p, const At& i) {
    return (T*)((char*)p + i.u * (int64_t)sizeof(T) + (uint32_t)(i.o * (uint32_t)sizeof(T)));
}

// A wave's part of a tile is FN fragments wide (gated: two half as wide ones) and at most four fragments high; a lane has eight neighbouring
// columns, and a pass takes as many rows as the lanes hold.
template <int FN, bool GATED> struct PartShape {
    static constexpr int CH = FN * 4, LPR = GATED ? CH / 4 : CH / 2;                 // fours of columns of sums in a row, lanes of a row
    static constexpr int RPP = 64 / LPR;                                             // rows of a pass
};

// A lane's first element in pass g over rows of `ld` elements; the part begins at element `first`.  The gradients of the operands have rows of K
// elements, up to 2^26: LONG has what grows with the pass in the uniform part, so that a lane's offset stays within the rows of one pass, at
// most 15 of them, under 2^32 bytes.  All other rows have 2^21 elements at most, of which 63 stay under 2^32 bytes: there the offset takes
// the pass as well (in the uniform part it would cost registers that the gated tile of 256 does not have).
template <int FN, bool GATED, bool LONG> LBA_HOST_DEVICE At lane_at(int64_t first, int64_t ld, int lane, int g) {
    typedef PartShape<FN, GATED> S;
    const uint32_t o = (uint32_t)(lane / S::LPR) * (uint32_t)ld + (uint32_t)(lane % S::LPR * 8);
    if constexpr (LONG) return {first + g * (S::RPP * ld), o};
    return {first, o + (uint32_t)g * (S::RPP * (uint32_t)ld)};
}

}  // namespace lba
#endif

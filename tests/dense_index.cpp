// Host build of the dense product's epilogue indices (csrc/lba_dense_index.h): the address of every element of a wave's part against
// 64-bit arithmetic, for rows up to the longest that the entry points take.  tests/test_dense_index_cpu.py compiles and runs it.
#include <cstdio>
#include <initializer_list>

#include "lba_dense_index.h"

static int failures = 0;

template <typename T, int FN, bool GATED, bool LONG> static void check_part(int rows, int64_t row0, int64_t col0, int64_t ld) {
    typedef lba::PartShape<FN, GATED> S;
    const T* const base = (const T*)((uintptr_t)1 << 40);       // never read
    for (int g = 0; g < rows / S::RPP; ++g)
        for (int lane = 0; lane < 64; ++lane) {
            const int64_t m = row0 + g * S::RPP + lane / S::LPR, n = col0 + lane % S::LPR * 8;
            const uintptr_t want = (uintptr_t)base + (uintptr_t)(m * ld + n) * sizeof(T);
            const lba::At i = lba::lane_at<FN, GATED, LONG>(row0 * ld + col0, ld, lane, g);
            if (((uintptr_t)lba::at(base, i) != want || i.u + (int64_t)i.o != m * ld + n) && ++failures < 10)
                std::printf("FAIL FN %d gated %d size %zu ld %lld row %lld column %lld: off by %lld bytes\n", FN, GATED, sizeof(T), (long long)ld,
                            (long long)m, (long long)n, (long long)((uintptr_t)lba::at(base, i) - want));
        }
}

template <typename T> static void check_all() {
    // dA and dB have rows of K elements with (rows + 64) (K + 64) <= 2^32, all other matrices of at most 2^21 and what fills a cache line
    const int64_t longest = ((int64_t)1 << 32) / 65 - 64;
    for (int64_t ld : {(int64_t)1, (int64_t)771, (int64_t)4096, (int64_t)17043520, (int64_t)17043522, ((int64_t)1 << 25) - 64, longest})
        for (int64_t row0 : {(int64_t)0, (int64_t)192, ((int64_t)1 << 30) - 64}) {
            check_part<T, 2, false, true>(32, row0, 0, ld);
            check_part<T, 4, false, true>(64, row0, 64, ld);
        }
    for (int64_t ld : {(int64_t)3, (int64_t)4096, (int64_t)1 << 20, ((int64_t)1 << 21) + 64})
        for (int64_t row0 : {(int64_t)0, ((int64_t)1 << 30) - 64}) {
            check_part<T, 2, false, false>(32, row0, 0, ld);
            check_part<T, 4, false, false>(64, row0, 64, ld);
            check_part<T, 2, true, false>(32, row0, 0, ld);
            check_part<T, 4, true, false>(64, row0, 64, ld);
        }
}

int main() {
    check_all<uint8_t>();
    check_all<uint16_t>();
    check_all<float>();
    std::printf(failures ? "%d failures\n" : "indices ok\n", failures);
    return failures != 0;
}

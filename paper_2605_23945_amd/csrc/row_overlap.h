// Overlaps of row-wise operands, a host check of the operators' entry points.
#pragma once
#include <stdint.h>

namespace pat {

// Whether any of m rows of wa bytes at a, lda bytes apart, has a byte in common with any of m rows of wb bytes at b, ldb apart (rows of one side do not overlap each other):
// row slices side by side in one buffer have none.
inline bool rows_overlap(const void *a, int64_t lda, int64_t wa, const void *b, int64_t ldb, int64_t wb, int64_t m)
{
    const int64_t d = (int64_t)((uintptr_t)b - (uintptr_t)a);
    if (d >= (m - 1) * lda + wa || -d >= (m - 1) * ldb + wb) return false;
    if (lda == ldb) {                                          // row 0 of b lies r behind a's row t, and lda - r in front of the next
        const int64_t t = d / lda - (d % lda < 0), r = d - t * lda;
        return (t > -m && t < m && r < wa) || (t + 1 > -m && t + 1 < m && lda - r < wb);
    }
    for (int64_t i = 0, j = 0; i < m && j < m;) {
        const int64_t from = d + j * ldb - i * lda;            // of b's row j behind a's row i
        if (from < wa && -from < wb) return true;
        if (from > 0) ++i; else ++j;
    }
    return false;
}

}  // namespace pat

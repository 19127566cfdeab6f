// Matrices in one memory (host code).
#pragma once

#include <stdint.h>

#include <algorithm>

namespace regot {

// Whether an element of S is one of dS, two matrices of n rows of m elements of b bytes at row distances ldS and ldD (which are no
// less than m).  Rows of one may lie between those of the other (columns of one wider matrix).
inline bool overlap(int64_t n, int64_t m, const void *S, int64_t ldS, const void *dS, int64_t ldD, int b)
{
    typedef __int128 wide;  // (addresses and row distances are anything)
    if (n == 0 || m == 0) return false;
    const wide row = (wide)m * b, stepS = (wide)ldS * b, stepD = (wide)ldD * b, S0 = (uintptr_t)S, D0 = (uintptr_t)dS;
    if (S0 >= D0 + (n - 1) * stepD + row || D0 >= S0 + (n - 1) * stepS + row) return false;
    // the rows of dS that begin at or before a row of S and after it; at equal distances it is the same for every row
    const auto meets = [&](wide at, int64_t i) { return i >= 0 && i < n && D0 + i * stepD < at + row && at < D0 + i * stepD + row; };
    if (stepS == stepD) {
        const wide from = D0 - S0;  // row i of S and row j of dS are (j - i) steps and `from` apart
        const wide j = from >= 0 ? -(from / stepD) : -from / stepD;
        for (wide d = j - 1; d <= j + 1; ++d) {
            const wide apart = from + d * stepD;
            if (d > -n && d < n && apart < row && -apart < row) return true;
        }
        return false;
    }
    for (int64_t i = 0; i < n; ++i) {
        const wide at = S0 + i * stepS;
        const wide j = at >= D0 ? (at - D0) / stepD : -1;
        const int64_t k = (int64_t)std::min<wide>(j, n);
        if (meets(at, k) || meets(at, k + 1)) return true;
    }
    return false;
}

}  // namespace regot

// A place among the offsets of consecutive ranges. Host and device code.
#pragma once

#include <stdint.h>

#include "mixed_order.h"

namespace sangam {

// The last of n + 1 offsets (not decreasing) that is at most x; -1: none. n up to 2^31 - 2.
SANGAM_HD inline int last_offset(const int32_t* indptr, int n, int64_t x) {
    int lo = -1, hi = n + 1;
    while (hi - 1 > lo) {
        const int mid = lo + int((uint32_t(hi) - uint32_t(lo)) / 2);  // (their sum or difference may not fit)
        if (indptr[mid] <= x) lo = mid;
        else hi = mid;
    }
    return lo;
}

}  // namespace sangam

// Which sequence holds a packed row.
#pragma once
#include "hyd_device.h"

namespace hyd {

// The sequence that holds packed row t, by a whole wave: s and its first row and end; false if t lies in none.  64 probes at a time.
__device__ __forceinline__ bool find_sequence(const int32_t* __restrict__ cu, int nseq, int t, int& s, int& first, int& end) {
    const int lane = threadIdx.x & 63;
    int lo = 0, n = nseq + 1;             // the last index i in [lo, lo + n) with cu[i] <= t, if there is one
    while (true) {
        const int step = (n + 63) / 64, i = lo + lane * step;
        const int c = lane * step < n ? cu[i] : 0x7fffffff;
        const int k = __popcll(__ballot(c <= t));
        if (k == 0) return false;
        lo += (k - 1) * step;
        n = min(step, n - (k - 1) * step);
        if (n == 1) {
            first = __shfl(c, k - 1, 64);
            break;
        }
    }
    if (lo >= nseq) return false;
    s = lo;
    end = cu[lo + 1];
    return true;
}

}  // namespace hyd

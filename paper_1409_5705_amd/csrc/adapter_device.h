// Device functions of the adapter calls' kernels.
#pragma once
#include "adapter.h"

namespace sfb {

// The request of row t, or -1 (empty requests are passed over: the last q with start[q] <= t).  By a whole wavefront: 64
// probes a step.
__device__ __forceinline__ int64_t request_of(const int64_t* start, int64_t requests, int64_t t, int lane)
{
    if (requests <= 0 || t < start[0] || t >= start[requests]) return -1;
    int64_t lo = 0, n = requests;                  // start[lo] <= t; the answer is in [lo, lo + n)
    while (n > 1) {
        const int64_t step = (n + 63) / 64, at = lane * step;
        const uint64_t below = __builtin_amdgcn_ballot_w64(at < n && start[lo + at] <= t);
        const int64_t k = 63 - __builtin_clzll(below | 1);
        lo += k * step;
        n = n - k * step < step ? n - k * step : step;
    }
    return lo;
}
__device__ __forceinline__ int rank_of(const int32_t* ranks, int rank, int64_t a)
{
    const int r = ranks ? ranks[a] : rank;
    return r < 0 ? 0 : r < rank ? r : rank;
}

}  // namespace sfb

// lamp_search.h -- a workgroup's place in a ragged batch (library-internal, device
// code).
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace lamp {
namespace {

// Sequence whose range of the non-decreasing starts f(0..S-1) holds x: the
// last s with f(s) <= x, by the whole wave, 64 places at once (each round is
// one load's latency).
template <class F>
__device__ __forceinline__ int last_at_most(int S, int64_t x, F f)
{
    const int lane = threadIdx.x & 63;
    int lo = 0, n = S;
    for (;;) {
        const int step = (n + 63) / 64;
        const int at = lo + lane * step;
        const uint64_t below = __ballot(lane == 0 || (lane * step < n && f(at) <= x));
        lo += (63 - __builtin_clzll(below)) * step;
        if (step == 1) return lo;
        n = S - lo < step ? S - lo : step;
    }
}

} // namespace
} // namespace lamp

// Packed sequences: which one a token or a tile belongs to.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

namespace mmee {

// The largest i < n with value(i) <= x, or -1; value ascends (where it does not, some number below n).  64 at a time, asked by a whole wave.
template <class F>
__device__ __forceinline__ int last_at_most(uint32_t n, int64_t x, F value)
{
    const uint32_t lane = threadIdx.x & 63;
    uint32_t lo = 0;
    bool first = true;
    while (n > 0) {
        const uint32_t step = (n + 63) / 64, at = lane * step;
        const uint64_t below = __ballot(at < n && value(lo + at) <= x);
        if (!below) return first ? -1 : (int)lo;
        const uint32_t last = 63 - __builtin_clzll(below);
        lo += last * step;
        n = step == 1 ? 0 : (n - last * step < step ? n - last * step : step);
        first = false;
    }
    return first ? -1 : (int)lo;
}

__device__ __forceinline__ int64_t within(int64_t x, int64_t lo, int64_t hi) { return x < lo ? lo : x > hi ? hi : x; }

}  // namespace mmee

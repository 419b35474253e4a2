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

// Join of the lanes up to a lane's own: their sum, or the largest of all.
template <class F>
__device__ __forceinline__ uint32_t scan_lanes(uint32_t x, F join)
{
    x = join(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x111, 0xf, 0xf, false));        // from 1, 2, 4, 8 lanes below within a row of 16
    x = join(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x112, 0xf, 0xf, false));
    x = join(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x114, 0xf, 0xf, false));
    x = join(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x118, 0xf, 0xf, false));
    x = join(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x142, 0xa, 0xf, false));        // row 0's last lane to row 1, row 2's to row 3
    return join(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x143, 0xc, 0xf, false));     // the lower half's last lane to the upper half
}

__device__ __forceinline__ uint32_t sums_below(uint32_t x)
{
    return scan_lanes(x, [](uint32_t a, uint32_t b) { return a + b; });
}

__device__ __forceinline__ uint32_t most_of_lanes(uint32_t x)
{
    return __builtin_amdgcn_readlane(scan_lanes(x, [](uint32_t a, uint32_t b) { return a > b ? a : b; }), 63);
}

}  // namespace mmee

// What the operators' translation units share with the rest of the library: its lock, its stream, its last error.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>
#include <mutex>

#include "../../include/mmee.h"

namespace mmee {

// Holds the library's lock for one call that enqueues kernels on the library's stream.
class Launching {
    std::unique_lock<std::mutex> held;

public:
    Launching();
    hipStream_t stream;
    int rc;                     // MMEE_OK, or MMEE_EDEVICE without a device
};

// MMEE_OK after a successful launch; otherwise keeps the error's text for mmee_strerror.  Under the lock.
int launched(const char *what);

// Blocks whose numbers agree modulo 8 run on one of the eight dies and share its L2: block `at` of n takes a number such that the
// blocks of a die are neighbours.  A permutation of 0 .. n-1 for any n.
__device__ __forceinline__ uint32_t by_die(uint32_t at, uint32_t n)
{
    const uint32_t die = at & 7, full = n >> 3, rest = n & 7;
    return die * full + (die < rest ? die : rest) + (at >> 3);
}

}  // namespace mmee

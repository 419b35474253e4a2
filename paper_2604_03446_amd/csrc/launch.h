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
    hipStream_t stream;
    hipError_t error = hipSuccess;      // the first of this call's launches.  (hipGetLastError would report, and clear, what the program met before.)

public:
    Launching();
    int rc;                             // MMEE_OK, or MMEE_EDEVICE without a device

    template <class Args>
    void run(void (*kernel)(Args), uint64_t blocks, uint32_t threads, Args args)
    {
        void *list[] = {&args};
        const hipError_t e = hipLaunchKernel(reinterpret_cast<const void *>(kernel), dim3((uint32_t)blocks), dim3(threads), list, 0, stream);
        if (error == hipSuccess) error = e;
    }

    int result(const char *what);       // MMEE_OK if every launch went well; otherwise keeps the error's text for mmee_strerror
};

// Blocks whose numbers agree modulo 8 run on one of the eight dies and share its L2: block `at` of n takes a number such that the
// blocks of a die are neighbours.  A permutation of 0 .. n-1 for any n.
__device__ __forceinline__ uint32_t by_die(uint32_t at, uint32_t n)
{
    const uint32_t die = at & 7, full = n >> 3, rest = n & 7;
    return die * full + (die < rest ? die : rest) + (at >> 3);
}

}  // namespace mmee

// Launches of blocks of another size than kBlock.
//
// Everything here lives in an unnamed namespace, like scram_device.h.

#pragma once

#include "scram_device.h"

namespace scram {
namespace {

// launch() for kernels of another block size: one wave, by default
template <uint32_t kThreads = 64, typename P>
hipError_t launch_wave(void (*kernel)(P), uint64_t blocks, hipStream_t st, hipEvent_t start, hipEvent_t stop,
                       const P& p)
{
    if (blocks == 0 || blocks > 0xFFFFFFFFull / kThreads) return hipErrorInvalidConfiguration;
    if (start || stop)
        hipExtLaunchKernelGGL(kernel, dim3(blocks), dim3(kThreads), 0, st, start, stop, 0, p);
    else
        hipLaunchKernelGGL(kernel, dim3(blocks), dim3(kThreads), 0, st, p);
    return hipGetLastError();
}

}  // namespace
}  // namespace scram

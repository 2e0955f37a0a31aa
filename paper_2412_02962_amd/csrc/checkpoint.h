// Internal interface of the 8-bit checkpoint kernels.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace pcpp {

// n values (whole groups of 32) of codes and scales as bf16, exactly.
hipError_t launch_checkpoint_load_bf16(const void* codes, const void* scales, void* y, int64_t n, hipStream_t s);

}  // namespace pcpp

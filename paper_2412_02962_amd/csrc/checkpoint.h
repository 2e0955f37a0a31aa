// Internal interface of the 8-bit checkpoint kernels.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace pcpp {

// What the feed-forward's backward pass needs before its products, in one
// launch; either part may be missing (n = 0, partial = null).
struct FfPrepare {
    const uint8_t* codes;   // n values (whole groups of 32) of x in 8 bits ...
    const uint8_t* scales;
    void* x;                // ... as bf16, exactly
    int64_t n;
    const void* dy;         // [rows, C] bf16, C % 64 == 0
    int64_t rows;
    int32_t C;
    float* partial;         // [column_partial_rows(rows)][C]: sums of dy over runs of rows
};
hipError_t launch_ff_prepare(const FfPrepare& p, hipStream_t s);

}  // namespace pcpp

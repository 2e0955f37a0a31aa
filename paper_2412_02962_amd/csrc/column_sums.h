// Sums over rows, for the gradients of biases and scales.  Rows are summed in
// a fixed order into float32 partial rows, these into the bf16 gradient: no
// atomics, so that a result does not depend on timing.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace pcpp {

// Partial rows of launch_column_partials for `rows` rows.
int column_partial_rows(int64_t rows);
// partial [column_partial_rows(rows)][C] float32 from x [rows][C] bf16, C % 8 == 0.
hipError_t launch_column_partials(const void* x, int64_t rows, int C, float* partial, hipStream_t s);
// out [C] bf16 = the sum of n partial rows.
hipError_t launch_sum_partials(const float* partial, int n, int C, void* out, hipStream_t s);

}  // namespace pcpp

// Sums over rows, for the gradients of biases and scales.  Rows are summed in
// a fixed order into float32 partial rows, these into the bf16 gradient: no
// atomics, so that a result does not depend on timing.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "common.h"

namespace pcpp {

// Up to two gradients [C] from their n partial rows [n][C] float32 (C = 0: none).
struct PartialSums {
    const float* partial[2];
    bf16* out[2];
    int32_t n[2], C[2];
};

constexpr int SUM_COLUMNS = 16;  // of a workgroup of 256; 16 threads share a column's rows
inline int partial_sum_blocks(const PartialSums& a) {
    return (a.C[0] + SUM_COLUMNS - 1) / SUM_COLUMNS + (a.C[1] + SUM_COLUMNS - 1) / SUM_COLUMNS;
}

// Workgroup `block` of partial_sum_blocks; lds: 16 x 17 floats.
__device__ __forceinline__ void sum_partials(const PartialSums& a, int block, float* lds) {
    const int first = (a.C[0] + SUM_COLUMNS - 1) / SUM_COLUMNS;
    const int s = block >= first;
    const int l = threadIdx.x & 15, r = threadIdx.x >> 4;
    const int c = (block - s * first) * SUM_COLUMNS + l, C = s ? a.C[1] : a.C[0], n = s ? a.n[1] : a.n[0];
    const float* partial = s ? a.partial[1] : a.partial[0];
    float t[4] = {0.f, 0.f, 0.f, 0.f};
    if (c < C) {
        int i = r;
        for (; i + 48 < n; i += 64)
#pragma unroll
            for (int u = 0; u < 4; ++u) t[u] += partial[(int64_t)(i + 16 * u) * C + c];
        for (; i < n; i += 16) t[0] += partial[(int64_t)i * C + c];
    }
    lds[17 * r + l] = (t[0] + t[1]) + (t[2] + t[3]);
    __syncthreads();
    if (r == 0 && c < C) {
        float v = 0.f;
#pragma unroll
        for (int i = 0; i < 16; ++i) v += lds[17 * i + l];
        (s ? a.out[1] : a.out[0])[c] = f32_to_bf16(v);
    }
}
hipError_t launch_sum_partials(const PartialSums& a, hipStream_t s);

// Partial rows of column_partials for `rows` rows, and its workgroups for C columns.
int column_partial_rows(int64_t rows);
inline int64_t column_partial_blocks(int64_t rows, int C) { return (int64_t)((C + 63) / 64) * column_partial_rows(rows); }

}  // namespace pcpp

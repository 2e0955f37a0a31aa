// Sums over rows, for the gradients of biases and scales.  Rows are summed in
// a fixed order into float32 partial rows, these into the bf16 gradient: no
// atomics, so that a result does not depend on timing.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "common.h"
#include "rows8.h"

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

// Sums of 64 columns of x over one of column_partial_rows(rows) runs of rows,
// eight columns a lane; a workgroup of 256, lds: COLUMN_LDS floats.
constexpr int COLUMN_LDS = 32 * (64 + 4);
__device__ __forceinline__ void column_partials(const bf16* x, int64_t rows, int C, float* partial, int64_t block,
                                                int runs, float* lds) {
    constexpr int kLaneRows = 256 / 8, LD = COLUMN_LDS / kLaneRows;
    const int l = threadIdx.x & 7, r = threadIdx.x >> 3;
    const int run = (int)(block / (C / 64)), c0 = 64 * (int)(block % (C / 64));
    const int64_t lo = rows * run / runs, hi = rows * (run + 1) / runs;
    float a[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) a[e] = 0.f;
    for (int64_t i = lo + r; i < hi; i += 4 * kLaneRows) {
        float v[4][8];
#pragma unroll
        for (int u = 0; u < 4; ++u) {
#pragma unroll
            for (int e = 0; e < 8; ++e) v[u][e] = 0.f;
            if (i + u * kLaneRows < hi) load8(x + (i + u * kLaneRows) * C + c0 + 8 * l, v[u]);
        }
#pragma unroll
        for (int u = 0; u < 4; ++u)
#pragma unroll
            for (int e = 0; e < 8; ++e) a[e] += v[u][e];
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) lds[LD * r + 8 * l + e] = a[e];
    __syncthreads();
    if (threadIdx.x < 64) {
        float t = 0.f;
#pragma unroll
        for (int i = 0; i < kLaneRows; ++i) t += lds[LD * i + threadIdx.x];
        partial[(int64_t)run * C + c0 + threadIdx.x] = t;
    }
}
// Its partial rows for `rows` rows, its workgroups for C columns (a multiple of
// 64), and a launch of its own.
int column_partial_rows(int64_t rows);
inline int column_partial_blocks(int64_t rows, int C) { return C / 64 * column_partial_rows(rows); }
hipError_t launch_column_partials(const bf16* x, int64_t rows, int C, float* partial, hipStream_t s);

}  // namespace pcpp

// Column sums (see column_sums.h).

#include "column_sums.h"

#include "common.h"
#include "rows8.h"

namespace pcpp {

namespace {

constexpr int kThreads = 256;
constexpr int kMaxPartials = 512;
constexpr int kLaneRows = kThreads / 8;  // 64 columns a workgroup, eight a lane

// Workgroup (x, y): columns 64 x .., the y-th of gridDim.y ranges of rows.
__global__ __launch_bounds__(kThreads) void column_partials(const bf16* x, int64_t rows, int C, float* partial) {
    __shared__ float lds[kLaneRows][64 + 4];
    const int l = threadIdx.x & 7, r = threadIdx.x >> 3;
    const int c = blockIdx.x * 64 + 8 * l;
    const int64_t lo = rows * blockIdx.y / gridDim.y, hi = rows * (blockIdx.y + 1) / gridDim.y;
    float a[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) a[e] = 0.f;
    if (c < C) {
        int64_t i = lo + r;
        for (; i + 3 * kLaneRows < hi; i += 4 * kLaneRows) {
            float v[4][8];
#pragma unroll
            for (int u = 0; u < 4; ++u) load8(x + (i + u * kLaneRows) * C + c, v[u]);
#pragma unroll
            for (int u = 0; u < 4; ++u)
#pragma unroll
                for (int e = 0; e < 8; ++e) a[e] += v[u][e];
        }
        for (; i < hi; i += kLaneRows) {
            float v[8];
            load8(x + i * C + c, v);
#pragma unroll
            for (int e = 0; e < 8; ++e) a[e] += v[e];
        }
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) lds[r][8 * l + e] = a[e];
    __syncthreads();
    const int n = blockIdx.x * 64 + threadIdx.x;
    if (threadIdx.x < 64 && n < C) {
        float t = 0.f;
#pragma unroll
        for (int i = 0; i < kLaneRows; ++i) t += lds[i][threadIdx.x];
        partial[(int64_t)blockIdx.y * C + n] = t;
    }
}

// The gradient from n partial rows: 16 channels a workgroup, 16 threads share a
// channel's rows.
__global__ __launch_bounds__(kThreads) void sum_partials(const float* partial, int n, int C, bf16* out) {
    __shared__ float lds[16][17];
    const int l = threadIdx.x & 15, r = threadIdx.x >> 4;
    const int c = blockIdx.x * 16 + l;
    float a[4] = {0.f, 0.f, 0.f, 0.f};
    if (c < C) {
        int i = r;
        for (; i + 48 < n; i += 64)
#pragma unroll
            for (int u = 0; u < 4; ++u) a[u] += partial[(int64_t)(i + 16 * u) * C + c];
        for (; i < n; i += 16) a[0] += partial[(int64_t)i * C + c];
    }
    lds[r][l] = (a[0] + a[1]) + (a[2] + a[3]);
    __syncthreads();
    if (r == 0 && c < C) {
        float t = 0.f;
#pragma unroll
        for (int i = 0; i < 16; ++i) t += lds[i][l];
        out[c] = f32_to_bf16(t);
    }
}

}  // namespace

int column_partial_rows(int64_t rows) {
    const int64_t n = (rows + 127) / 128;
    return (int)(n < kMaxPartials ? n : kMaxPartials);
}

hipError_t launch_column_partials(const void* x, int64_t rows, int C, float* partial, hipStream_t s) {
    column_partials<<<dim3((C + 63) / 64, column_partial_rows(rows)), kThreads, 0, s>>>((const bf16*)x, rows, C, partial);
    return hipGetLastError();
}

hipError_t launch_sum_partials(const float* partial, int n, int C, void* out, hipStream_t s) {
    sum_partials<<<(C + 15) / 16, kThreads, 0, s>>>(partial, n, C, (bf16*)out);
    return hipGetLastError();
}

}  // namespace pcpp

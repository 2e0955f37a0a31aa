// Root-mean-square norm with the residual's addition, and its backward pass.
//   pcpp_rms_norm           s = x + addend;  y = s * rstd * gamma,
//                           rstd = (mean s^2 + eps)^-1/2; y in bf16 and/or in
//                           8 bits with scales
//   pcpp_rms_norm_backward  n = s * rstd, w = dy * gamma:
//                           ds = ds_in + rstd (w - n mean(w n)),
//                           dgamma = sum over rows of dy * n
//
// Both are bound by the memory: a row is read once, held in registers (eight
// channels a lane and chunk, float32) between its sum and its use, and
// written once.  One wavefront takes a row of up to 2048 channels, four of a
// workgroup a longer one (or one of so few rows that the chip would idle).
// The backward pass recomputes rstd from the row that it reads anyway, so
// nothing but s is kept from the forward pass.
//
// Measured: forward 2 x 1280 5.4 us (a launch), 115200 x 640 with a float32
// stream and an addend 155 us (885 MB, 5.7 TB/s: a copy of 1 GiB reaches 5.2,
// part of the stream comes from the last-level cache), 8192 x 1280 with 8 bits
// too 41 us (168 MB, two calls); backward 777 x 1088 9.2 us (two launches, the
// second sums dgamma), 57600 x 640 100 us (516 MB, 5.2 TB/s).

#include <stdint.h>

#include <type_traits>

#include "../../include/pcpp.h"
#include "args.h"
#include "column_sums.h"
#include "common.h"
#include "eight_bit.h"
#include "kernels.h"
#include "rows8.h"

#define PCPP_EXPORT extern "C" __attribute__((visibility("default")))

namespace pcpp {

namespace {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / 64;
constexpr int kMaxC = 8192;
constexpr int kMaxBlocks = 1 << 20;
constexpr int kGradBlocks = 1024;  // most partial sums of dgamma

struct RmsParams {
    const void* x;        // [rows, C] the stream
    const bf16* addend;   // or null
    const bf16* gamma;
    void* sum;            // x + addend in the stream's type, or null
    bf16* y;              // or null
    uint8_t* codes;       // or null
    uint8_t* scales;
    int32_t rows, C;
    float eps;
};

struct RmsBackwardParams {
    const void* s;
    const bf16* gamma;
    const bf16* dy;
    const void* ds_in;    // or null
    void* ds;
    float* partial;       // [gridDim.x][C], or null
    int32_t rows, C;
    float eps;
};

// The sum of v over the wavefronts of a row (WPR of them: one, or the whole
// workgroup), in every lane.
template <int WPR>
__device__ __forceinline__ float row_sum(float v, float* lds) {
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) v += __shfl_xor(v, d);
    if constexpr (WPR > 1) {
        __syncthreads();  // the previous sum has been read
        if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
        __syncthreads();
        v = 0.f;
#pragma unroll
        for (int w = 0; w < WPR; ++w) v += lds[w];
    }
    return v;
}

// Chunk j of a lane: channels 8 * (lane of the row + 64 WPR j).
template <typename T, int WPR, int NCH>
__global__ __launch_bounds__(kThreads) void rms_norm(RmsParams p) {
    __shared__ float lds[kWaves];
    constexpr int RPB = kWaves / WPR;
    const int wave = threadIdx.x >> 6;
    const int c0 = 8 * (WPR == 1 ? (int)(threadIdx.x & 63) : (int)threadIdx.x);
    for (int64_t row = (int64_t)blockIdx.x * RPB + wave / WPR; row < p.rows; row += (int64_t)gridDim.x * RPB) {
        const int64_t at = row * p.C;
        float s[NCH][8];
        float sum = 0.f;
#pragma unroll
        for (int j = 0; j < NCH; ++j) {
            const int c = c0 + 512 * WPR * j;
#pragma unroll
            for (int e = 0; e < 8; ++e) s[j][e] = 0.f;
            if (c < p.C) {
                load8((const T*)p.x + at + c, s[j]);
                if (p.addend != nullptr) {
                    float r[8];
                    load8(p.addend + at + c, r);
#pragma unroll
                    for (int e = 0; e < 8; ++e) s[j][e] += r[e];
                }
            }
#pragma unroll
            for (int e = 0; e < 8; ++e) sum = __builtin_fmaf(s[j][e], s[j][e], sum);
        }
        const float rstd = 1.f / sqrtf(row_sum<WPR>(sum, lds) / (float)p.C + p.eps);
#pragma unroll
        for (int j = 0; j < NCH; ++j) {
            const int c = c0 + 512 * WPR * j;
            if (c >= p.C) continue;  // C % 32 == 0 with codes: a group's lanes stay together
            if (p.sum != nullptr) store8((T*)p.sum + at + c, s[j]);
            float g[8];
            load8(p.gamma + c, g);
            // n = s rstd first, at most sqrt(C): rstd gamma may be no float32
#pragma unroll
            for (int e = 0; e < 8; ++e) s[j][e] = s[j][e] * rstd * g[e];
            if (p.y != nullptr) store8(p.y + at + c, s[j]);
            if (p.codes != nullptr) {
                int scale;
                *(u32x2*)(p.codes + at + c) = to_eight_bits(s[j], scale);
                if ((threadIdx.x & 3) == 0) p.scales[(at + c) / EIGHT_GROUP] = (uint8_t)scale;
            }
        }
    }
}

template <typename T, int WPR, int NCH>
__global__ __launch_bounds__(kThreads) void rms_norm_backward(RmsBackwardParams p) {
    __shared__ float lds[kWaves];
    constexpr int RPB = kWaves / WPR;
    const int wave = threadIdx.x >> 6;
    const int c0 = 8 * (WPR == 1 ? (int)(threadIdx.x & 63) : (int)threadIdx.x);
    float dg[NCH][8];
#pragma unroll
    for (int j = 0; j < NCH; ++j)
#pragma unroll
        for (int e = 0; e < 8; ++e) dg[j][e] = 0.f;
    for (int64_t row = (int64_t)blockIdx.x * RPB + wave / WPR; row < p.rows; row += (int64_t)gridDim.x * RPB) {
        const int64_t at = row * p.C;
        float s[NCH][8], d[NCH][8];
        float sq = 0.f, dot = 0.f;
#pragma unroll
        for (int j = 0; j < NCH; ++j) {
            const int c = c0 + 512 * WPR * j;
#pragma unroll
            for (int e = 0; e < 8; ++e) s[j][e] = d[j][e] = 0.f;
            if (c < p.C) {
                load8((const T*)p.s + at + c, s[j]);
                load8(p.dy + at + c, d[j]);
                float g[8];
                load8(p.gamma + c, g);
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    sq = __builtin_fmaf(s[j][e], s[j][e], sq);
                    dot = __builtin_fmaf(d[j][e] * g[e], s[j][e], dot);
                }
            }
        }
        const float rstd = 1.f / sqrtf(row_sum<WPR>(sq, lds) / (float)p.C + p.eps);
        // mean(w n); rstd (w - n mean(w n)) by n and w, not by rstd^3 or dy rstd,
        // which overflow for small rows where eps lets them
        const float mean = rstd * (row_sum<WPR>(dot, lds) / (float)p.C);
#pragma unroll
        for (int j = 0; j < NCH; ++j) {
            const int c = c0 + 512 * WPR * j;
            if (c >= p.C) continue;
            float g[8], o[8];
            load8(p.gamma + c, g);
#pragma unroll
            for (int e = 0; e < 8; ++e) o[e] = 0.f;
            if (p.ds_in != nullptr) load8((const T*)p.ds_in + at + c, o);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float n = s[j][e] * rstd;
                dg[j][e] = __builtin_fmaf(d[j][e], n, dg[j][e]);
                o[e] = __builtin_fmaf(rstd, __builtin_fmaf(-mean, n, d[j][e] * g[e]), o[e]);
            }
            store8((T*)p.ds + at + c, o);
        }
    }
    if (p.partial == nullptr) return;
    if constexpr (WPR == 1) {  // the four wavefronts' rows, added in their order
        extern __shared__ __attribute__((aligned(16))) float acc[];
        for (int w = 0; w < kWaves; ++w) {
            if (wave == w) {
#pragma unroll
                for (int j = 0; j < NCH; ++j) {
                    const int c = c0 + 512 * j;
                    if (c >= p.C) continue;
                    if (w > 0) {
                        float o[8];
                        load8(acc + c, o);
#pragma unroll
                        for (int e = 0; e < 8; ++e) dg[j][e] += o[e];
                    }
                    if (w < kWaves - 1)
                        store8(acc + c, dg[j]);
                    else
                        store8(p.partial + (int64_t)blockIdx.x * p.C + c, dg[j]);
                }
            }
            __syncthreads();
        }
    } else {
#pragma unroll
        for (int j = 0; j < NCH; ++j) {
            const int c = c0 + 512 * WPR * j;
            if (c < p.C) store8(p.partial + (int64_t)blockIdx.x * p.C + c, dg[j]);
        }
    }
}

// Wavefronts per row: one up to 2048 channels (what its registers hold) unless
// the rows are so few that four a row still leave compute units without work.
// One and four, bf16: 256 x 1280 forward 5.6 and 5.3 us, backward 9.1 and 8.4;
// 2048 x 1280 backward 11.3 and 14.8 (more partial sums of dgamma), 8192 x 640
// forward 7.8 and 10.5.
int waves_per_row(int64_t rows, int C) { return C > 2048 || (C > 512 && rows <= 256) ? kWaves : 1; }

// f(template arguments) for the wavefronts and chunks of a row of C channels.
template <typename F>
void with_shape(int wpr, int C, F f) {
    const int n = (C + 512 * wpr - 1) / (512 * wpr);
    using std::integral_constant;
    if (wpr == 1) {
        if (n == 1) f(integral_constant<int, 1>(), integral_constant<int, 1>());
        else if (n == 2) f(integral_constant<int, 1>(), integral_constant<int, 2>());
        else if (n == 3) f(integral_constant<int, 1>(), integral_constant<int, 3>());
        else f(integral_constant<int, 1>(), integral_constant<int, 4>());
    } else {
        if (n == 1) f(integral_constant<int, kWaves>(), integral_constant<int, 1>());
        else if (n == 2) f(integral_constant<int, kWaves>(), integral_constant<int, 2>());
        else if (n == 3) f(integral_constant<int, kWaves>(), integral_constant<int, 3>());
        else f(integral_constant<int, kWaves>(), integral_constant<int, 4>());
    }
}

int64_t row_blocks(int64_t rows, int wpr) { return (rows * wpr + kWaves - 1) / kWaves; }

int grad_blocks(int64_t rows, int C) {
    const int64_t b = row_blocks(rows, waves_per_row(rows, C));
    return (int)(b < kGradBlocks ? b : kGradBlocks);
}

}  // namespace

}  // namespace pcpp

using namespace pcpp;

static int check_rows(int64_t rows, int32_t channels, float eps, int32_t dtype) {
    if (rows < 1 || rows > ((int64_t)1 << 24) || channels < 1 || !(eps > 0.f)) return PCPP_EINVAL;
    if (dtype != PCPP_DTYPE_F32 && dtype != PCPP_DTYPE_BF16) return PCPP_ENOTSUP;
    return channels % 8 != 0 || channels > kMaxC ? PCPP_ENOTSUP : PCPP_OK;
}

PCPP_EXPORT int pcpp_rms_norm(int64_t rows, int32_t channels, float eps, int32_t dtype, const void* x,
                              const void* addend, const void* gamma, void* sum_out, void* y, void* codes, void* scales,
                              void* stream) {
    const int st = check_rows(rows, channels, eps, dtype);
    if (st != PCPP_OK) return st;
    if (codes && channels % EIGHT_GROUP != 0) return PCPP_ENOTSUP;
    if (!x || !gamma || (!y && !codes) || (codes == nullptr) != (scales == nullptr)) return PCPP_EINVAL;
    const void* ptrs[] = {x, addend, gamma, sum_out, y, codes};
    for (const void* p : ptrs)
        if (!aligned_to(p, 16)) return PCPP_EINVAL;
    const int64_t n = rows * channels, size = dtype == PCPP_DTYPE_F32 ? 4 : 2;
    // the sum may replace x: every element is read and written by one lane
    const Range out[] = {{y, 2 * n}, {codes, n}, {scales, n / EIGHT_GROUP}, {sum_out, size * n}};
    const Range in[] = {{addend, 2 * n}, {gamma, 2 * (int64_t)channels}, {x, size * n}};
    if (outputs_overlap(out, sum_out == x ? 3 : 4, in, 3)) return PCPP_EINVAL;
    if (sum_out == x && outputs_overlap(out + 3, 1, in, 2)) return PCPP_EINVAL;
    const RmsParams p = {x, (const bf16*)addend, (const bf16*)gamma, sum_out, (bf16*)y, (uint8_t*)codes,
                         (uint8_t*)scales, (int32_t)rows, channels, eps};
    const int wpr = waves_per_row(rows, channels);
    const int64_t blocks = row_blocks(rows, wpr);
    const unsigned grid = (unsigned)(blocks < kMaxBlocks ? blocks : kMaxBlocks);
    with_shape(wpr, channels, [&](auto w, auto c) {
        if (dtype == PCPP_DTYPE_F32)
            rms_norm<float, w(), c()><<<grid, kThreads, 0, (hipStream_t)stream>>>(p);
        else
            rms_norm<bf16, w(), c()><<<grid, kThreads, 0, (hipStream_t)stream>>>(p);
    });
    return hipGetLastError() == hipSuccess ? PCPP_OK : PCPP_EHIP;
}

PCPP_EXPORT size_t pcpp_rms_norm_backward_workspace_size(int64_t rows, int32_t channels) {
    if (check_rows(rows, channels, 1.f, PCPP_DTYPE_F32) != PCPP_OK) return 0;
    return (size_t)grad_blocks(rows, channels) * channels * sizeof(float);
}

PCPP_EXPORT int pcpp_rms_norm_backward(int64_t rows, int32_t channels, float eps, int32_t dtype, const void* s,
                                       const void* gamma, const void* dy, const void* ds_in, void* ds, void* dgamma,
                                       void* workspace, size_t ws_bytes, void* stream) {
    const int st = check_rows(rows, channels, eps, dtype);
    if (st != PCPP_OK) return st;
    if (!s || !gamma || !dy || !ds) return PCPP_EINVAL;
    const void* ptrs[] = {s, gamma, dy, ds_in, ds, dgamma};
    for (const void* p : ptrs)
        if (!aligned_to(p, 16)) return PCPP_EINVAL;
    const int blocks = grad_blocks(rows, channels);
    const int64_t need = (int64_t)blocks * channels * 4;
    if (dgamma && (!workspace || ws_bytes < (size_t)need)) return PCPP_EWORKSPACE;
    if (dgamma && !aligned_to(workspace, 16)) return PCPP_EINVAL;
    const int64_t n = rows * channels, size = dtype == PCPP_DTYPE_F32 ? 4 : 2, cb = 2 * (int64_t)channels;
    // ds may replace ds_in: every element is read and written by one lane
    const Range out[] = {{ds, size * n}, {dgamma, cb}, {dgamma ? workspace : nullptr, need}};
    const Range in[] = {{s, size * n}, {gamma, cb}, {dy, 2 * n}, {ds == ds_in ? nullptr : ds_in, size * n}};
    if (outputs_overlap(out, 3, in, 4)) return PCPP_EINVAL;
    const RmsBackwardParams p = {s, (const bf16*)gamma, (const bf16*)dy, ds_in, ds,
                                 dgamma ? (float*)workspace : nullptr, (int32_t)rows, channels, eps};
    with_shape(waves_per_row(rows, channels), channels, [&](auto w, auto c) {
        const size_t lds = w() == 1 ? channels * sizeof(float) : 0;
        if (dtype == PCPP_DTYPE_F32)
            rms_norm_backward<float, w(), c()><<<blocks, kThreads, lds, (hipStream_t)stream>>>(p);
        else
            rms_norm_backward<bf16, w(), c()><<<blocks, kThreads, lds, (hipStream_t)stream>>>(p);
    });
    if (hipGetLastError() != hipSuccess) return PCPP_EHIP;
    if (!dgamma) return PCPP_OK;
    const PartialSums sums = {{p.partial, nullptr}, {(bf16*)dgamma, nullptr}, {blocks, 0}, {channels, 0}};
    return launch_sum_partials(sums, (hipStream_t)stream) == hipSuccess ? PCPP_OK : PCPP_EHIP;
}

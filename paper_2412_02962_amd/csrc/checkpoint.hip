// 8-bit activation checkpoints: rows to codes and scales, and back.
//   pcpp_checkpoint_save, pcpp_checkpoint_load
// Both are bound by the memory: eight channels a lane, a group's scale by two
// permutations within its four lanes, several chunks in flight.  Measured, both
// ways: 2048 x 640 bf16 9.8 us (two launches), 16384 x 5120 float32 133 us
// (671 MB, 5.0 TB/s; 131 before the values were quieted).

#include <stdint.h>

#include "../../include/pcpp.h"
#include "args.h"
#include "checkpoint.h"
#include "common.h"
#include "eight_bit.h"
#include "rows8.h"

#define PCPP_EXPORT extern "C" __attribute__((visibility("default")))

namespace pcpp {

namespace {

constexpr int kThreads = CHUNK_THREADS, kUnroll = CHUNK_UNROLL;

// Both kernels see the rows as one run of n8 chunks of eight channels (a
// row's channels are a multiple of 32, so no group crosses its end).
template <typename T>
__global__ __launch_bounds__(kThreads) void checkpoint_save(const T* x, uint8_t* codes, uint8_t* scales, int64_t n8) {
    const int64_t i0 = (int64_t)blockIdx.x * (kThreads * kUnroll) + threadIdx.x;
    float v[kUnroll][8];
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
        const int64_t i = i0 + u * kThreads;
        if (i < n8) load8(x + i * 8, v[u]);
    }
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
        const int64_t i = i0 + u * kThreads;
        if (i >= n8) break;  // n8 is a multiple of four: a group's lanes leave together
#pragma unroll
        for (int e = 0; e < 8; ++e) v[u][e] = quieted(v[u][e]);  // the caller's bits, of no arithmetic
        int scale;
        *(u32x2*)(codes + i * 8) = to_eight_bits(v[u], scale);
        if ((threadIdx.x & 3) == 0) scales[i >> 2] = (uint8_t)scale;
    }
}

template <typename T>
__global__ __launch_bounds__(kThreads) void checkpoint_load(const uint8_t* codes, const uint8_t* scales, T* y,
                                                            int64_t n8) {
    load_chunks(codes, scales, y, n8, blockIdx.x);
}

}  // namespace

}  // namespace pcpp

using namespace pcpp;

// Sizes, type and pointers of both calls; `x` the rows in full precision.
static int check_checkpoint(int64_t rows, int32_t channels, int32_t dtype, const void* x, const void* codes,
                            const void* scales) {
    if (rows < 1 || rows > ((int64_t)1 << 24) || channels < 1) return PCPP_EINVAL;
    if (dtype != PCPP_DTYPE_F32 && dtype != PCPP_DTYPE_BF16) return PCPP_ENOTSUP;
    if (channels % EIGHT_GROUP != 0 || channels > (1 << 16)) return PCPP_ENOTSUP;
    if (!x || !codes || !scales || !aligned_to(x, 16) || !aligned_to(codes, 16)) return PCPP_EINVAL;
    const int64_t n = rows * channels;
    if (n > ((int64_t)1 << 36)) return PCPP_EINVAL;  // a launch has fewer than 2^32 threads
    const Range all[] = {{x, n * (dtype == PCPP_DTYPE_F32 ? 4 : 2)}, {codes, n}, {scales, n / EIGHT_GROUP}};
    return outputs_overlap(all, 3, nullptr, 0) ? PCPP_EINVAL : PCPP_OK;
}

PCPP_EXPORT int pcpp_checkpoint_save(int64_t rows, int32_t channels, int32_t dtype, const void* x, void* codes,
                                     void* scales, void* stream) {
    const int st = check_checkpoint(rows, channels, dtype, x, codes, scales);
    if (st != PCPP_OK) return st;
    const int64_t n8 = rows * channels / 8;
    if (dtype == PCPP_DTYPE_F32)
        checkpoint_save<<<chunk_blocks(n8), kThreads, 0, (hipStream_t)stream>>>((const float*)x, (uint8_t*)codes,
                                                                             (uint8_t*)scales, n8);
    else
        checkpoint_save<<<chunk_blocks(n8), kThreads, 0, (hipStream_t)stream>>>((const bf16*)x, (uint8_t*)codes,
                                                                             (uint8_t*)scales, n8);
    return hipGetLastError() == hipSuccess ? PCPP_OK : PCPP_EHIP;
}

PCPP_EXPORT int pcpp_checkpoint_load(int64_t rows, int32_t channels, int32_t dtype, const void* codes,
                                     const void* scales, void* y, void* stream) {
    const int st = check_checkpoint(rows, channels, dtype, y, codes, scales);
    if (st != PCPP_OK) return st;
    const int64_t n = rows * channels;
    const unsigned blocks = chunk_blocks(n / 8);
    if (dtype == PCPP_DTYPE_BF16)
        checkpoint_load<<<blocks, kThreads, 0, (hipStream_t)stream>>>((const uint8_t*)codes, (const uint8_t*)scales,
                                                                      (bf16*)y, n / 8);
    else
        checkpoint_load<<<blocks, kThreads, 0, (hipStream_t)stream>>>((const uint8_t*)codes, (const uint8_t*)scales,
                                                                      (float*)y, n / 8);
    return hipGetLastError() == hipSuccess ? PCPP_OK : PCPP_EHIP;
}

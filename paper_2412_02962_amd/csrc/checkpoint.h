// 8-bit rows read back, for the checkpoint kernels and the feed-forward's
// backward pass.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "column_sums.h"
#include "common.h"
#include "eight_bit.h"
#include "rows8.h"

namespace pcpp {

// Rows as one run of n8 chunks of eight channels, CHUNK_UNROLL a thread.
constexpr int CHUNK_THREADS = 256, CHUNK_UNROLL = 4;
inline unsigned chunk_blocks(int64_t n8) {
    return (unsigned)((n8 + CHUNK_THREADS * CHUNK_UNROLL - 1) / (CHUNK_THREADS * CHUNK_UNROLL));
}

template <typename T>
__device__ __forceinline__ void load_chunks(const uint8_t* codes, const uint8_t* scales, T* y, int64_t n8,
                                            int64_t block) {
    const int64_t i0 = block * (CHUNK_THREADS * CHUNK_UNROLL) + threadIdx.x;
    u32x2 c[CHUNK_UNROLL];
    int s[CHUNK_UNROLL];
#pragma unroll
    for (int u = 0; u < CHUNK_UNROLL; ++u) {
        const int64_t i = i0 + u * CHUNK_THREADS;
        if (i < n8) {
            c[u] = *(const u32x2*)(codes + i * 8);
            s[u] = scales[i >> 2];
        }
    }
#pragma unroll
    for (int u = 0; u < CHUNK_UNROLL; ++u) {
        const int64_t i = i0 + u * CHUNK_THREADS;
        if (i >= n8) break;
        const float f = eight_value(s[u]);
        const f32x4 a = from_e4m3(c[u][0]), b = from_e4m3(c[u][1]);
        float v[8];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            v[e] = a[e] * f;
            v[4 + e] = b[e] * f;
        }
        store8(y + i * 8, v);
    }
}

// What the gradients' products need besides the gate's gradient: workgroups of
// its launch do this after its own.  Either part may be missing (n = 0, partial
// = null).
struct FfPrepare {
    const uint8_t* codes;   // n values (whole groups of 32) of x in 8 bits ...
    const uint8_t* scales;
    bf16* x;                // ... as bf16, exactly
    int64_t n;
    const bf16* dy;         // [rows, C], C % 64 == 0
    int64_t rows;
    int32_t C;
    float* partial;         // [column_partial_rows(rows)][C]: sums of dy over runs of rows
    int32_t runs;           // column_partial_rows(rows)
    int32_t sum_blocks;     // workgroups of the sums; those of x follow
};
inline int64_t prepare_blocks(const FfPrepare& p) { return p.sum_blocks + (p.n > 0 ? chunk_blocks(p.n / 8) : 0); }
// lds: COLUMN_LDS floats.
__device__ __forceinline__ void prepare_block(const FfPrepare& p, int64_t block, float* lds) {
    if (block < p.sum_blocks)
        column_partials(p.dy, p.rows, p.C, p.partial, block, p.runs, lds);
    else
        load_chunks(p.codes, p.scales, p.x, p.n / 8, block - p.sum_blocks);
}

}  // namespace pcpp

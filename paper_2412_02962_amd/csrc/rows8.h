// Eight consecutive channels of a row between memory and float registers.
#pragma once

#include "common.h"

namespace pcpp {

__device__ __forceinline__ void load8(const float* p, float (&v)[8]) {
    const f32x4 a = *(const f32x4*)p, b = *(const f32x4*)(p + 4);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        v[i] = a[i];
        v[4 + i] = b[i];
    }
}

__device__ __forceinline__ void load8(const bf16* p, float (&v)[8]) {
    const bf16x8 a = *(const bf16x8*)p;
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = bf16_to_f32(a[i]);
}

__device__ __forceinline__ void store8(float* p, const float (&v)[8]) {
    *(f32x4*)p = f32x4{v[0], v[1], v[2], v[3]};
    *(f32x4*)(p + 4) = f32x4{v[4], v[5], v[6], v[7]};
}

__device__ __forceinline__ void store8(bf16* p, const float (&v)[8]) {
    bf16x8 a;
#pragma unroll
    for (int i = 0; i < 8; ++i) a[i] = f32_to_bf16(v[i]);
    *(bf16x8*)p = a;
}

}  // namespace pcpp

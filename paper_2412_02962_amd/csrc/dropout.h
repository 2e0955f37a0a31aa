// Dropout's mask: a function of the generator's state and an element's place,
// computed where it is needed and never stored.
//
// Eight consecutive elements share one block of Philox 4x32-10 (J. Salmon et
// al., Parallel random numbers: as easy as 1, 2, 3, SC 2011): key = the seed,
// counter = (place / 8, stream).  Element e takes the 16 bits e of the block,
// from the lowest, and is kept where they are at least round(65536 p): the
// factor 65536 / (65536 - round(65536 p)) makes the mean of a kept value exact
// for the p that is applied, within 2^-17 of the one asked for.  (A block per
// four elements, 32 bits each, costs twice the multiplications.)
#pragma once

#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include "common.h"

namespace pcpp {

// A call's dropout.  least = 0: everything is kept and the state is not read.
struct Dropout {
    const uint64_t* rng;  // device: seed, first stream
    uint64_t draw;        // added to the first stream
    uint32_t least;       // 0 .. 65536
    float factor;
};

// The dropout of probability p, finite and in [0, 1].
inline Dropout make_dropout(float p, const void* rng, uint64_t draw) {
    const uint32_t least = (uint32_t)lrint((double)p * 65536.0);
    return Dropout{(const uint64_t*)rng, draw, least, least < 65536 ? 65536.0f / (float)(65536 - least) : 0.f};
}

// What a wavefront reads of it once.
struct DropoutKey {
    uint32_t key0, key1, stream0, stream1;
};
__device__ __forceinline__ DropoutKey dropout_key(const Dropout& d) {
    if (d.least == 0) return DropoutKey{};
    const uint64_t seed = d.rng[0], stream = d.rng[1] + d.draw;
    return DropoutKey{(uint32_t)seed, (uint32_t)(seed >> 32), (uint32_t)stream, (uint32_t)(stream >> 32)};
}

__device__ __forceinline__ u32x4 philox(const DropoutKey& k, uint64_t block) {
    uint32_t c0 = (uint32_t)block, c1 = (uint32_t)(block >> 32), c2 = k.stream0, c3 = k.stream1;
    uint32_t k0 = k.key0, k1 = k.key1;
#pragma unroll
    for (int r = 0; r < 10; ++r) {
        const uint64_t a = (uint64_t)c0 * 0xD2511F53u, b = (uint64_t)c2 * 0xCD9E8D57u;
        c0 = (uint32_t)(b >> 32) ^ c1 ^ k0;
        c1 = (uint32_t)b;
        c2 = (uint32_t)(a >> 32) ^ c3 ^ k1;
        c3 = (uint32_t)a;
        k0 += 0x9E3779B9u;
        k1 += 0xBB67AE85u;
    }
    return u32x4{c0, c1, c2, c3};
}

// The eight elements of block `block`: as they are, or 0 (whatever they were).
__device__ __forceinline__ void keep8(const Dropout& d, const DropoutKey& k, uint64_t block, float (&v)[8]) {
    const u32x4 w = philox(k, block);
    // compared in the upper halves, where a least of 2^16 would be lost: no
    // element is kept then
    const uint32_t least = d.least << 16, none = d.least >> 16;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const uint32_t bits = e & 1 ? w[e >> 1] : w[e >> 1] << 16;
        v[e] = bits >= least ? v[e] : 0.f;
    }
    if (none)
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = 0.f;
}

// The same, what is kept scaled.
__device__ __forceinline__ void drop8(const Dropout& d, const DropoutKey& k, uint64_t block, float (&v)[8]) {
    keep8(d, k, block, v);
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] *= d.factor;
}

}  // namespace pcpp

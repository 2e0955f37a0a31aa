// Internal interface of the gated feed-forward's products.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "common.h"

namespace pcpp {

// What follows a product Y = X W^T in its epilogue.
enum FfEpilogue {
    FF_STORE,    // out = Y + bias, bf16
    FF_GATE,     // W's rows hold value and gate: out = v act(g), and v, g in 8 bits
    FF_GATE_GRAD // Y = dh: out = [dh act(g), dh v act'(g)], h = v act(g), sums of out's columns
};

// X [M, K] and W [N, K], or stored the other way round: x_t: X is [K, M]
// in memory (rows of ldx elements), w_t: W is [K, N].
struct FfProduct {
    const bf16* x;
    const bf16* w;
    int64_t ldx, ldw;
    int32_t x_t, w_t;
    int32_t M, N, K;      // FF_GATE: N = F outputs, W has 2F rows
    int32_t epilogue;     // FfEpilogue
    int32_t act;          // PCPP_ACT_*
    bf16* out;            // [M, N], FF_GATE_GRAD: [M, 2N]; null: not wanted (FF_GATE_GRAD)
    const bf16* bias;     // [rows of W] or null
    uint8_t* codes;       // [M, 2N] e4m3 of value and gate (FF_GATE: written, or null; FF_GATE_GRAD: read)
    uint8_t* scales;      // [M, 2N / 32]
    bf16* h;              // FF_GATE_GRAD: [M, N] or null
    float* partial;       // FF_GATE_GRAD: [ff_partial_rows(M)][2N] sums of out over rows, or null
    int32_t tiles, n_xcd, per_xcd;  // set by the launch
};
int ff_partial_rows(int64_t M);
// A product with X along the contraction (w_t as the epilogue has it: only
// FF_GATE_GRAD's W lies across it).
hipError_t launch_ff_product(const FfProduct& p, hipStream_t s);
// Up to three products of FF_STORE with w_t = 1, those with x_t = 1 first, in one launch.
hipError_t launch_ff_products(const FfProduct* p, int n, hipStream_t s);

}  // namespace pcpp

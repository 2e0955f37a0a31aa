// Internal interface of the gated feed-forward's products.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "checkpoint.h"
#include "column_sums.h"
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
    float* partial;       // FF_GATE_GRAD: [ff_partial_rows(p)][2N] sums of out over rows, or null
    // Set by the launch: the pieces that the contraction is worked in, their
    // float32 sums [pieces][M][N], tiles x pieces, and how they go to the XCDs.
    int32_t pieces;
    float* part;
    int32_t items, n_xcd, per_xcd;
};
int ff_partial_rows(const FfProduct& p);  // of a product's sizes and epilogue
// FF_GATE, and FF_STORE of what it wrote, on at most FF_SKINNY_ROWS rows of X,
// both operands along the contraction (ff_skinny.hip); launch_ff_product calls
// it for these.  On at most FF_SPLIT_ROWS FF_GATE's out and FF_STORE's x are
// [2][M][F], two bf16 whose sum is h.
constexpr int FF_SPLIT_ROWS = 8;
constexpr int FF_SKINNY_ROWS = 16;
hipError_t launch_ff_skinny(const FfProduct& p, int cus, hipStream_t s);
int ff_skinny_outputs(const FfProduct& p, int cus);  // of a workgroup
// A product of FF_STORE or FF_GATE with both operands along the contraction, one
// of FF_GATE_GRAD with W across it (the launch also does `pre`), and up to three
// of FF_STORE with W across it (which also does `sums`).  part: ff_part_floats of
// the same products, or of these and others.
hipError_t launch_ff_product(FfProduct p, float* part, hipStream_t s);
hipError_t launch_ff_gate_grad(FfProduct p, const FfPrepare& pre, hipStream_t s);
hipError_t launch_ff_products(const FfProduct* p, int n, float* part, const PartialSums& sums, hipStream_t s);
int64_t ff_part_floats(const FfProduct* p, int n);
// What they run on with `cus` compute units (0: the current device's): the
// tile, and the pieces in p.
void ff_plan(FfProduct* p, int n, int cus, int32_t* tile_rows, int32_t* tile_outputs);

}  // namespace pcpp

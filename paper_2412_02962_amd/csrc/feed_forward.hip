// The gated feed-forward block and its backward pass (C ABI).
//   pcpp_gated_ff           [v, g] = x W1^T + b1;  h = v act(g);  y = h W2^T + b2:
//                           both projections, the activation and the product
//                           in one kernel (which also writes the 8-bit
//                           checkpoint of v and g), then the down projection
//   pcpp_gated_ff_backward  one product dh = dy W2 whose epilogue reads the
//                           checkpoint and leaves dpre = [dv, dg], h and the
//                           columns' sums, then dx = dpre W1, dW1 = dpre^T x
//                           and dW2 = dy^T h

#include "feed_forward.h"

#include "../../include/pcpp.h"
#include "args.h"
#include "checkpoint.h"
#include "column_sums.h"
#include "eight_bit.h"
#include "kernels.h"

#define PCPP_EXPORT extern "C" __attribute__((visibility("default")))

namespace pcpp {

namespace {

constexpr int kMaxC = 8192, kMaxF = 1 << 16;

int check_geom(const pcpp_ff_geom_t* g) {
    if (!g || g->reserved != 0 || g->tokens < 1 || g->tokens > ((int64_t)1 << 24) || g->channels < 1 || g->ff_inner < 1)
        return PCPP_EINVAL;
    if (g->act != PCPP_ACT_GELU && g->act != PCPP_ACT_SILU) return PCPP_ENOTSUP;
    if (g->channels % 64 != 0 || g->channels > kMaxC || g->ff_inner % 64 != 0 || g->ff_inner > kMaxF) return PCPP_ENOTSUP;
    // a launch has fewer than 2^32 threads
    return g->tokens * g->ff_inner > ((int64_t)1 << 36) ? PCPP_EINVAL : PCPP_OK;
}

// Byte offsets within a workspace, every part 256-byte aligned.
struct Layout {
    size_t size = 0;
    size_t add(int64_t bytes) {
        const size_t at = size;
        size += ((size_t)bytes + 255) & ~(size_t)255;
        return at;
    }
};

// The products of both passes, without their pointers.
FfProduct product(const pcpp_ff_geom_t& g, FfEpilogue epilogue, int64_t M, int64_t N, int64_t K, int x_t, int w_t) {
    FfProduct p = {};
    p.M = (int32_t)M;
    p.N = (int32_t)N;
    p.K = (int32_t)K;
    p.ldx = x_t ? M : K;
    p.ldw = w_t ? N : K;
    p.x_t = x_t;
    p.w_t = w_t;
    p.epilogue = epilogue;
    p.act = g.act;
    return p;
}
FfProduct up_of(const pcpp_ff_geom_t& g) { return product(g, FF_GATE, g.tokens, g.ff_inner, g.channels, 0, 0); }
FfProduct down_of(const pcpp_ff_geom_t& g) { return product(g, FF_STORE, g.tokens, g.channels, g.ff_inner, 0, 0); }
FfProduct gate_grad_of(const pcpp_ff_geom_t& g) {
    return product(g, FF_GATE_GRAD, g.tokens, g.ff_inner, g.channels, 0, 1);
}
FfProduct w1_grad_of(const pcpp_ff_geom_t& g) {
    return product(g, FF_STORE, 2 * (int64_t)g.ff_inner, g.channels, g.tokens, 1, 1);
}
FfProduct w2_grad_of(const pcpp_ff_geom_t& g) { return product(g, FF_STORE, g.channels, g.ff_inner, g.tokens, 1, 1); }
FfProduct x_grad_of(const pcpp_ff_geom_t& g) {
    return product(g, FF_STORE, g.tokens, g.channels, 2 * (int64_t)g.ff_inner, 0, 1);
}

struct ForwardLayout : Layout {
    size_t h, part;
    explicit ForwardLayout(const pcpp_ff_geom_t& g) {
        h = add((g.tokens <= FF_SPLIT_ROWS ? 4 : 2) * g.tokens * g.ff_inner);
        const FfProduct down = down_of(g);
        part = add(4 * ff_part_floats(&down, 1));
    }
};

struct BackwardLayout : Layout {
    size_t x, dpre, h, sums1, sums2, part;
    explicit BackwardLayout(const pcpp_ff_geom_t& g) {
        const int64_t M = g.tokens, C = g.channels, F = g.ff_inner;
        x = add(2 * M * C);
        dpre = add(4 * M * F);
        h = add(2 * M * F);
        sums1 = add((int64_t)ff_partial_rows(gate_grad_of(g)) * 2 * F * 4);
        sums2 = add((int64_t)column_partial_rows(M) * C * 4);
        const FfProduct p[] = {w1_grad_of(g), w2_grad_of(g), x_grad_of(g)};
        part = add(4 * ff_part_floats(p, 3));
    }
};

bool all_aligned(const Range* r, int n) {
    for (int i = 0; i < n; ++i)
        if (!aligned_to(r[i].p, 16)) return false;
    return true;
}

}  // namespace

}  // namespace pcpp

using namespace pcpp;

PCPP_EXPORT size_t pcpp_gated_ff_workspace_size(const pcpp_ff_geom_t* g) {
    if (check_geom(g) != PCPP_OK) return 0;
    return ForwardLayout(*g).size;
}

PCPP_EXPORT int pcpp_gated_ff_plan(const pcpp_ff_geom_t* g, int32_t which, int32_t cus, int32_t* tile_rows,
                                   int32_t* tile_outputs, int32_t* pieces) {
    const int st = check_geom(g);
    if (st != PCPP_OK) return st;
    if (which < PCPP_FF_UP || which > PCPP_FF_X_GRAD || cus < 0) return PCPP_EINVAL;
    if (cus == 0 && device_cus() == 0) return PCPP_EHIP;
    FfProduct p[] = {w1_grad_of(*g), w2_grad_of(*g), x_grad_of(*g)};
    int n = 3, at = which - PCPP_FF_W1_GRAD;
    if (which < PCPP_FF_W1_GRAD) {
        p[0] = which == PCPP_FF_UP ? up_of(*g) : which == PCPP_FF_DOWN ? down_of(*g) : gate_grad_of(*g);
        n = 1;
        at = 0;
    }
    int32_t rows, outputs;
    ff_plan(p, n, cus, &rows, &outputs);
    if (tile_rows) *tile_rows = rows;
    if (tile_outputs) *tile_outputs = outputs;
    if (pieces) *pieces = p[at].pieces;
    return PCPP_OK;
}

PCPP_EXPORT int pcpp_gated_ff(const pcpp_ff_geom_t* g, const pcpp_ff_weights_t* w, const void* x, void* y,
                              void* pre_codes, void* pre_scales, void* workspace, size_t ws_bytes, void* stream) {
    const int st = check_geom(g);
    if (st != PCPP_OK) return st;
    if (!w || !w->ff1_w || !w->ff2_w || !x || !y || (pre_codes == nullptr) != (pre_scales == nullptr)) return PCPP_EINVAL;
    const int64_t M = g->tokens, C = g->channels, F = g->ff_inner;
    const ForwardLayout l(*g);
    if (!workspace || ws_bytes < l.size) return PCPP_EWORKSPACE;
    const Range in[] = {{x, 2 * M * C}, {w->ff1_w, 4 * F * C}, {w->ff1_b, 4 * F}, {w->ff2_w, 2 * C * F}, {w->ff2_b, 2 * C}};
    const Range out[] = {{y, 2 * M * C}, {workspace, (int64_t)l.size}, {pre_codes, 2 * M * F}, {pre_scales, 2 * M * F / EIGHT_GROUP}};
    if (!all_aligned(in, 5) || !all_aligned(out, 3) || outputs_overlap(out, 4, in, 5)) return PCPP_EINVAL;
    const hipStream_t s = (hipStream_t)stream;
    bf16* h = (bf16*)((char*)workspace + l.h);
    FfProduct up = up_of(*g);
    up.x = (const bf16*)x;
    up.w = (const bf16*)w->ff1_w;
    up.out = h;
    up.bias = (const bf16*)w->ff1_b;
    up.codes = (uint8_t*)pre_codes;
    up.scales = (uint8_t*)pre_scales;
    if (launch_ff_product(up, nullptr, s) != hipSuccess) return PCPP_EHIP;
    FfProduct down = down_of(*g);
    down.x = h;
    down.w = (const bf16*)w->ff2_w;
    down.out = (bf16*)y;
    down.bias = (const bf16*)w->ff2_b;
    return launch_ff_product(down, (float*)((char*)workspace + l.part), s) == hipSuccess ? PCPP_OK : PCPP_EHIP;
}

PCPP_EXPORT size_t pcpp_gated_ff_backward_workspace_size(const pcpp_ff_geom_t* g) {
    return check_geom(g) == PCPP_OK ? BackwardLayout(*g).size : 0;
}

PCPP_EXPORT int pcpp_gated_ff_backward(const pcpp_ff_geom_t* g, const pcpp_ff_weights_t* w, const void* x,
                                       const void* x_scales, const void* pre_codes, const void* pre_scales,
                                       const void* dy, void* dx, const pcpp_ff_grads_t* grads, void* workspace,
                                       size_t ws_bytes, void* stream) {
    const int st = check_geom(g);
    if (st != PCPP_OK) return st;
    const pcpp_ff_grads_t none = {};
    const pcpp_ff_grads_t& d = grads ? *grads : none;
    if (!w || !w->ff1_w || !w->ff2_w || !x || !pre_codes || !pre_scales || !dy) return PCPP_EINVAL;
    if (!dx && !d.ff1_w && !d.ff1_b && !d.ff2_w && !d.ff2_b) return PCPP_EINVAL;
    const int64_t M = g->tokens, C = g->channels, F = g->ff_inner;
    const BackwardLayout l(*g);
    if (!workspace || ws_bytes < l.size) return PCPP_EWORKSPACE;
    const Range in[] = {{x, (x_scales ? 1 : 2) * M * C}, {pre_codes, 2 * M * F}, {dy, 2 * M * C}, {w->ff1_w, 4 * F * C},
                        {w->ff2_w, 2 * C * F}, {x_scales, M * C / EIGHT_GROUP}, {pre_scales, 2 * M * F / EIGHT_GROUP}};
    const Range out[] = {{dx, 2 * M * C}, {d.ff1_w, 4 * F * C}, {d.ff1_b, 4 * F}, {d.ff2_w, 2 * C * F}, {d.ff2_b, 2 * C},
                         {workspace, (int64_t)l.size}};
    if (!all_aligned(in, 5) || !all_aligned(out, 6) || outputs_overlap(out, 6, in, 7)) return PCPP_EINVAL;
    const hipStream_t s = (hipStream_t)stream;
    char* ws = (char*)workspace;
    bf16 *dpre = (bf16*)(ws + l.dpre), *h = (bf16*)(ws + l.h);
    float *sums1 = (float*)(ws + l.sums1), *sums2 = (float*)(ws + l.sums2);
    FfPrepare pre = {};
    const bf16* x16 = (const bf16*)x;
    if (d.ff1_w && x_scales) {
        x16 = (const bf16*)(ws + l.x);
        pre.codes = (const uint8_t*)x;
        pre.scales = (const uint8_t*)x_scales;
        pre.x = (bf16*)(ws + l.x);
        pre.n = M * C;
    }
    if (d.ff2_b) {
        pre.dy = (const bf16*)dy;
        pre.rows = M;
        pre.C = (int32_t)C;
        pre.partial = sums2;
        pre.runs = column_partial_rows(M);
        pre.sum_blocks = column_partial_blocks(M, (int)C);
    }
    if (dx || d.ff1_w || d.ff1_b || d.ff2_w) {
        FfProduct p = gate_grad_of(*g);
        p.x = (const bf16*)dy;
        p.w = (const bf16*)w->ff2_w;
        p.out = dx || d.ff1_w ? dpre : nullptr;
        p.codes = (uint8_t*)const_cast<void*>(pre_codes);
        p.scales = (uint8_t*)const_cast<void*>(pre_scales);
        p.h = d.ff2_w ? h : nullptr;
        p.partial = d.ff1_b ? sums1 : nullptr;
        if (launch_ff_gate_grad(p, pre, s) != hipSuccess) return PCPP_EHIP;
    } else if (launch_column_partials(pre.dy, M, (int)C, sums2, s) != hipSuccess) {  // ff2_b alone
        return PCPP_EHIP;
    }
    PartialSums sums = {};
    if (d.ff1_b) {
        sums.partial[0] = sums1;
        sums.out[0] = (bf16*)d.ff1_b;
        sums.n[0] = ff_partial_rows(gate_grad_of(*g));
        sums.C[0] = (int32_t)(2 * F);
    }
    if (d.ff2_b) {
        sums.partial[1] = sums2;
        sums.out[1] = (bf16*)d.ff2_b;
        sums.n[1] = column_partial_rows(M);
        sums.C[1] = (int32_t)C;
    }
    FfProduct group[3] = {};
    int n = 0;
    if (d.ff1_w) {
        FfProduct& p = group[n++] = w1_grad_of(*g);
        p.x = dpre;
        p.w = x16;
        p.out = (bf16*)d.ff1_w;
    }
    if (d.ff2_w) {
        FfProduct& p = group[n++] = w2_grad_of(*g);
        p.x = (const bf16*)dy;
        p.w = h;
        p.out = (bf16*)d.ff2_w;
    }
    if (dx) {
        FfProduct& p = group[n++] = x_grad_of(*g);
        p.x = dpre;
        p.w = (const bf16*)w->ff1_w;
        p.out = (bf16*)dx;
    }
    return launch_ff_products(group, n, (float*)(ws + l.part), sums, s) == hipSuccess ? PCPP_OK : PCPP_EHIP;
}

// The gated feed-forward's products on few tokens (see feed_forward.h): at
// most 16 rows of X, both operands along the contraction.
//
// What bounds them is the weights' way from memory, each read once (1 token,
// 1280 x 5120: 39 MB), and the latency of a load, of which a loop over tiles
// in LDS pays one per tile.  So a workgroup takes few rows of W (32 outputs'
// values and gates, or 16 outputs) and its eight wavefronts an eighth of the
// contraction each; W goes straight from memory into the MFMA's operand
// registers, a run of k-steps in flight at a time, as does X, which the L2
// holds.  The wavefronts' sums meet in LDS.  A compute unit takes in some 40
// bytes a cycle, so that half as many outputs go to a workgroup as long as each
// still has a compute unit to itself (FF_GATE, without the checkpoint, whose
// groups are 32 outputs: 16; FF_STORE: 8, half the matrix unit's rows).  1 token:
// 640 x 2560 11.9 -> 10.5 us, 1280 x 5120 16.9 -> 15.0; with more workgroups than
// compute units it is the other way, 4096 x 8192 58 -> 61.
//
// Between the two products of up to eight tokens, h's values are sums of two
// bf16, 16 significant bits, so that y is rounded once: the matrix unit takes
// 16 tokens, the second halves go where the other eight would be.  They cost
// their way into the compute unit, 8 tokens 1280 x 5120 19.0 us, 9 tokens 17.3;
// error against float64 0.0016, not 0.0023.
//
// More than 16 tokens take the tiles: 16 tokens 1280 x 5120 19.6 us, 17 by tiles 23.5;
// two columns of tokens here would read twice as much of X per compute unit.
//
// 1 token 1280 x 5120: 8.3 and 6.0 to 7.0 us, 26 and 13 MB, where a launch alone is
// about 5 and the bytes take 5.0 and 2.5; other splits of the contraction (16
// wavefronts, 4 to 20 k-steps in flight) were within 5 % of it at 640 x 2560,
// 1280 x 5120 and 2048 x 5504.

#include "eight_bit.h"
#include "feed_forward.h"
#include "ff_act.h"

namespace pcpp {

namespace {

constexpr int kWaves = 8, kThreads = 64 * kWaves;

__device__ __forceinline__ f32x4 mfma16(bf16x8 a, bf16x8 b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}

// BNO outputs: W rows n0 .. and, FF_GATE, N further on.
template <int EPI, int ACT, int BNO>
__global__ __launch_bounds__(kThreads) void ff_skinny(FfProduct p) {
    constexpr int NV = (BNO + 15) / 16, NB = EPI == FF_GATE ? 2 * NV : NV;  // blocks of 16 W rows: values, gates
    constexpr int U = 8;  // k-steps in flight
    __shared__ f32x4 sums[kWaves][NB][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int lr = lane & 15, lq = lane >> 4;
    const int n0 = blockIdx.x * BNO;

    const bf16* w[NB];
#pragma unroll
    for (int i = 0; i < NB; ++i)
        w[i] = p.w + (int64_t)(n0 + 16 * (i % NV) + (i >= NV ? p.N : 0) + lr % BNO) * p.ldw + 8 * lq;
    // FF_STORE of at most eight tokens: lanes 8 .. 15 take the second halves of
    // the sums that X's values are, [2][M][K].
    const bool two = EPI != FF_GATE && p.M <= FF_SPLIT_ROWS;
    const int row = two ? lr & 7 : lr;
    const bool there = row < p.M;
    const bf16* x = p.x + (int64_t)(there ? row + (two && lr >= 8 ? p.M : 0) : 0) * p.ldx + 8 * lq;
    f32x4 acc[NB];
#pragma unroll
    for (int i = 0; i < NB; ++i) acc[i] = f32x4{0.f, 0.f, 0.f, 0.f};

    const int steps = p.K / 32;  // K % 64 == 0
    const int s1 = steps * (wave + 1) / kWaves;
    for (int s = steps * wave / kWaves; s < s1; s += U) {
        bf16x8 wv[U][NB], xv[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const bool in = s + u < s1;  // past the end: zeros
#pragma unroll
            for (int i = 0; i < NB; ++i) {
                wv[u][i] = bf16x8{};
                if (in && lr < BNO) wv[u][i] = *(const bf16x8*)(w[i] + 32 * (s + u));
            }
            xv[u] = bf16x8{};
            if (in && there) xv[u] = *(const bf16x8*)(x + 32 * (s + u));
        }
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int i = 0; i < NB; ++i) acc[i] = mfma16(wv[u][i], xv[u], acc[i]);
    }

    // acc[i][e]: W row 16 i + 4 lq + e, token (or half of its sum) lr
#pragma unroll
    for (int i = 0; i < NB; ++i) sums[wave][i][lane] = acc[i];
    __syncthreads();
    const int n = threadIdx.x % BNO, m = threadIdx.x / BNO;  // output, token
    auto total = [&](int i, int row) {  // of row `row` of block i, the wavefronts in their order
        float t = 0.f, second = 0.f;
#pragma unroll
        for (int k = 0; k < kWaves; ++k) {
            t += sums[k][i][16 * (row >> 2) + m][row & 3];
            if (two) second += sums[k][i][16 * (row >> 2) + 8 + (m & 7)][row & 3];
        }
        // an infinite weight times a second half, zero or of the other sign, is
        // no part of the sum
        return two && is_finite(t) ? t + second : t;
    };
    if (m >= 16 || m >= p.M) return;  // a group's 32 lanes together (BNO = 32)
    if constexpr (EPI == FF_GATE) {
        float v = total(n >> 4, n & 15), g = total(NV + (n >> 4), n & 15);
        if (p.bias != nullptr) {
            v += bf16_to_f32(p.bias[n0 + n]);
            g += bf16_to_f32(p.bias[p.N + n0 + n]);
        }
        if (BNO == EIGHT_GROUP && p.codes != nullptr) {
            const int64_t at = (int64_t)m * 2 * p.N + n0 + n;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const float a = h ? g : v;
                float top = finite_abs(a);
#pragma unroll
                for (int d = 1; d < 32; d <<= 1) top = fmaxf(top, __shfl_xor(top, d));
                const int scale = eight_scale(top);
                p.codes[at + h * p.N] = (uint8_t)to_e4m3(eight_scaled(a, eight_inverse(scale)), 0.f, 0.f, 0.f);
                if (n == 0) p.scales[(at + h * p.N) / EIGHT_GROUP] = (uint8_t)scale;
            }
        }
        const float h = v * ff_act<ACT>(g);
        const bf16 high = f32_to_bf16(h);
        bf16* out = p.out + (int64_t)m * p.N + n0 + n;
        out[0] = high;
        if (p.M <= FF_SPLIT_ROWS) {  // nothing is left of what is infinite in bf16
            const float top = bf16_to_f32(high);
            out[(int64_t)p.M * p.N] = f32_to_bf16(fabsf(top) < INFINITY ? h - top : 0.f);
        }
    } else {
        float v = total(0, n);
        if (p.bias != nullptr) v += bf16_to_f32(p.bias[n0 + n]);
        p.out[(int64_t)m * p.N + n0 + n] = f32_to_bf16(v);
    }
}

}  // namespace

int ff_skinny_outputs(const FfProduct& p, int cus) {
    const int few = p.epilogue == FF_GATE ? 16 : 8;
    return p.N / few <= cus && (p.epilogue != FF_GATE || p.codes == nullptr) ? few : 2 * few;
}

hipError_t launch_ff_skinny(const FfProduct& p, int cus, hipStream_t s) {
    const int outputs = ff_skinny_outputs(p, cus);
    auto run = [&](auto kernel) { kernel<<<p.N / outputs, kThreads, 0, s>>>(p); };
    const bool silu = p.act == PCPP_ACT_SILU;
    if (p.epilogue == FF_STORE)
        run(outputs == 8 ? ff_skinny<FF_STORE, 0, 8> : ff_skinny<FF_STORE, 0, 16>);
    else if (outputs == 16)
        run(silu ? ff_skinny<FF_GATE, PCPP_ACT_SILU, 16> : ff_skinny<FF_GATE, PCPP_ACT_GELU, 16>);
    else
        run(silu ? ff_skinny<FF_GATE, PCPP_ACT_SILU, 32> : ff_skinny<FF_GATE, PCPP_ACT_GELU, 32>);
    return hipGetLastError();
}

}  // namespace pcpp

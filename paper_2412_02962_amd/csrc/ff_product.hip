// The gated feed-forward's products on 16x16x32 bf16 MFMAs (see
// feed_forward.h): Y = X W^T with either operand stored along or across the
// contraction, and the activation, its derivative and the 8-bit checkpoint in
// the epilogue.

#include "eight_bit.h"
#include "feed_forward.h"
#include "ff_act.h"

namespace pcpp {

namespace {

constexpr int BM = 128, BN = 128, BK = 32;
constexpr int kThreads = 256;
constexpr int LDK = BK + 8;  // elements per LDS row

__device__ __forceinline__ f32x4 mfma16(bf16x8 a, bf16x8 b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}

// Rows [r0, r0 + 128) of an operand, 32 of its contraction from k0, into LDS
// rows of LDK; zeros outside its `rows` rows and K.
template <bool T, typename RowOf>
__device__ __forceinline__ void stage(const bf16* x, int64_t ld, int K, int k0, RowOf row_of, bf16* lds) {
    const int tid = threadIdx.x;
#pragma unroll
    for (int q = 0; q < 2; ++q) {
        const int i = tid + kThreads * q;
        bf16x8 v = {};
        if constexpr (!T) {
            const int r = i >> 2, c = 8 * (i & 3);
            const int row = row_of(r);
            if (row >= 0 && k0 + c < K) v = *(const bf16x8*)(x + (int64_t)row * ld + k0 + c);
            *(bf16x8*)(lds + r * LDK + c) = v;
        } else {
            const int k = i >> 4, r = 8 * (i & 15);
            const int row = row_of(r);
            if (row >= 0 && k0 + k < K) v = *(const bf16x8*)(x + (int64_t)(k0 + k) * ld + row);
#pragma unroll
            for (int e = 0; e < 8; ++e) lds[(r + e) * LDK + k] = v[e];
        }
    }
}

template <bool XT, bool WT, int EPI>
__global__ __launch_bounds__(kThreads) void ff_product(FfProduct p) {
    __shared__ __attribute__((aligned(16))) bf16 xs[BM * LDK], ws[BN * LDK];
    constexpr int BNO = EPI == FF_GATE ? BN / 2 : BN;  // outputs of a tile
    const int n_tiles = (p.N + BNO - 1) / BNO;
    const int m0 = (int)(blockIdx.x / n_tiles) * BM, n0 = (int)(blockIdx.x % n_tiles) * BNO;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int wm = wave & 1, wn = wave >> 1;
    const int lr = lane & 15, lq = lane >> 4;
    auto x_row = [&](int r) { return m0 + r < p.M ? m0 + r : -1; };
    // FF_GATE: of every 64 rows of a tile 32 are values, 32 their gates
    auto w_row = [&](int r) {
        if constexpr (EPI == FF_GATE) {
            const int n = n0 + 32 * (r >> 6) + (r & 31);
            return n < p.N ? n + ((r & 32) ? p.N : 0) : -1;
        } else {
            return n0 + r < p.N ? n0 + r : -1;
        }
    };
    f32x4 acc[4][4];
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
    for (int k0 = 0; k0 < p.K; k0 += BK) {
        __syncthreads();
        stage<XT>(p.x, p.ldx, p.K, k0, x_row, xs);
        stage<WT>(p.w, p.ldw, p.K, k0, w_row, ws);
        __syncthreads();
        bf16x8 xv[4], wv[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            xv[j] = *(const bf16x8*)(xs + (64 * wm + 16 * j + lr) * LDK + 8 * lq);
            wv[j] = *(const bf16x8*)(ws + (64 * wn + 16 * j + lr) * LDK + 8 * lq);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) acc[i][j] = mfma16(wv[i], xv[j], acc[i][j]);
    }
    // acc[i][j][e]: W row 64 wn + 16 i + 4 lq + e, X row 64 wm + 16 j + lr
    auto to_bf16 = [](f32x4 v) { return bf16x4{(bf16)v[0], (bf16)v[1], (bf16)v[2], (bf16)v[3]}; };
    auto widen = [](bf16x4 v) { return f32x4{(float)v[0], (float)v[1], (float)v[2], (float)v[3]}; };
    if constexpr (EPI == FF_STORE) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int n = n0 + 64 * wn + 16 * i + 4 * lq;
            if (n >= p.N) continue;
            f32x4 b = {0.f, 0.f, 0.f, 0.f};
            if (p.bias) b = widen(*(const bf16x4*)(p.bias + n));
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int m = m0 + 64 * wm + 16 * j + lr;
                if (m < p.M) *(bf16x4*)(p.out + (int64_t)m * p.N + n) = to_bf16(acc[i][j] + b);
            }
        }
    } else if constexpr (EPI == FF_GATE) {
        const int nb = n0 + 32 * wn;  // this wavefront's 32 outputs, one group of the checkpoint
        if (nb >= p.N) return;
        if (p.bias) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const f32x4 b = widen(*(const bf16x4*)(p.bias + (i >= 2 ? p.N : 0) + nb + 16 * (i & 1) + 4 * lq));
#pragma unroll
                for (int j = 0; j < 4; ++j) acc[i][j] += b;
            }
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int m = m0 + 64 * wm + 16 * j + lr;
            if (p.codes) {
#pragma unroll
                for (int g = 0; g < 2; ++g) {  // value, gate
                    float top = 0.f;
#pragma unroll
                    for (int i = 0; i < 2; ++i)
#pragma unroll
                        for (int e = 0; e < 4; ++e) top = fmaxf(top, finite_abs(acc[2 * g + i][j][e]));
                    top = fmaxf(top, __shfl_xor(top, 16));
                    top = fmaxf(top, __shfl_xor(top, 32));
                    const int scale = eight_scale(top);
                    const float inv = eight_inverse(scale);
                    const int64_t at = (int64_t)m * 2 * p.N + g * p.N + nb;
                    if (m < p.M) {
#pragma unroll
                        for (int i = 0; i < 2; ++i) {
                            const f32x4 a = acc[2 * g + i][j];
                            *(uint32_t*)(p.codes + at + 16 * i + 4 * lq) =
                                to_e4m3(eight_scaled(a[0], inv), eight_scaled(a[1], inv), eight_scaled(a[2], inv),
                                        eight_scaled(a[3], inv));
                        }
                        if (lq == 0) p.scales[at / EIGHT_GROUP] = (uint8_t)scale;
                    }
                }
            }
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                f32x4 v;
#pragma unroll
                for (int e = 0; e < 4; ++e) v[e] = acc[i][j][e] * ff_act(p.act, acc[2 + i][j][e]);
                if (m < p.M) *(bf16x4*)(p.out + (int64_t)m * p.N + nb + 16 * i + 4 * lq) = to_bf16(v);
            }
        }
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int n = n0 + 64 * wn + 16 * i + 4 * lq;
            if (n >= p.N) continue;  // a wavefront's 64 columns are all inside or all outside
            f32x4 sv = {0.f, 0.f, 0.f, 0.f}, sg = sv;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int m = m0 + 64 * wm + 16 * j + lr;
                if (m >= p.M) continue;
                const int64_t at = (int64_t)m * 2 * p.N + n;
                const f32x4 v = from_e4m3(*(const uint32_t*)(p.codes + at)) * eight_value(p.scales[at / EIGHT_GROUP]);
                const f32x4 g = from_e4m3(*(const uint32_t*)(p.codes + at + p.N)) *
                                eight_value(p.scales[(at + p.N) / EIGHT_GROUP]);
                f32x4 dv, dg, h;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    float da;
                    const float a = ff_act(p.act, g[e], &da);
                    dv[e] = acc[i][j][e] * a;
                    dg[e] = acc[i][j][e] * v[e] * da;
                    h[e] = v[e] * a;
                }
                sv += dv;
                sg += dg;
                if (p.out) {
                    *(bf16x4*)(p.out + at) = to_bf16(dv);
                    *(bf16x4*)(p.out + at + p.N) = to_bf16(dg);
                }
                if (p.h) *(bf16x4*)(p.h + (int64_t)m * p.N + n) = to_bf16(h);
            }
            if (p.partial) {
#pragma unroll
                for (int d = 1; d < 16; d <<= 1)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        sv[e] += __shfl_xor(sv[e], d);
                        sg[e] += __shfl_xor(sg[e], d);
                    }
                if (lr == 0) {
                    float* at = p.partial + (int64_t)((m0 >> 6) + wm) * 2 * p.N + n;
                    *(f32x4*)at = sv;
                    *(f32x4*)(at + p.N) = sg;
                }
            }
        }
    }
}

}  // namespace

int ff_partial_rows(int64_t M) { return (int)(2 * ((M + BM - 1) / BM)); }

hipError_t launch_ff_product(const FfProduct& p, hipStream_t s) {
    const int bno = p.epilogue == FF_GATE ? BN / 2 : BN;
    const unsigned grid = (unsigned)((int64_t)((p.M + BM - 1) / BM) * ((p.N + bno - 1) / bno));
    if (p.epilogue == FF_GATE)
        ff_product<false, false, FF_GATE><<<grid, kThreads, 0, s>>>(p);
    else if (p.epilogue == FF_GATE_GRAD)
        ff_product<false, true, FF_GATE_GRAD><<<grid, kThreads, 0, s>>>(p);
    else if (p.x_t)
        ff_product<true, true, FF_STORE><<<grid, kThreads, 0, s>>>(p);
    else if (p.w_t)
        ff_product<false, true, FF_STORE><<<grid, kThreads, 0, s>>>(p);
    else
        ff_product<false, false, FF_STORE><<<grid, kThreads, 0, s>>>(p);
    return hipGetLastError();
}

}  // namespace pcpp

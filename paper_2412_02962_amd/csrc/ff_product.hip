// The gated feed-forward's products (see feed_forward.h): Y = X W^T with
// either operand stored along or across the contraction, on 32x32x16 bf16
// MFMAs, with the activation, its derivative and the 8-bit checkpoint in the
// epilogue.

#include "eight_bit.h"
#include "feed_forward.h"
#include "ff_act.h"
#include "rows8.h"

namespace pcpp {

namespace {

constexpr int KT = 64;  // contraction per tile
constexpr int WAVES = 4;
constexpr int THREADS = 64 * WAVES;

typedef __attribute__((address_space(3))) void* lptr;
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) s16x4* s16x4_lds;

// 16 bytes per lane into LDS at lds + 16 lane, from byte voff of the buffer
// (zeros past its end).  Inline assembly, so that the compiler does not wait
// for loads in flight before every LDS read: the kernel orders them itself.
__device__ __forceinline__ void dma16(u32x4 buffer, uint32_t voff, uint32_t lds) {
    asm volatile("s_nop 0\n\tbuffer_load_dwordx4 %0, %1, 0 offen lds" ::"v"(voff), "s"(buffer), "{m0}"(lds) : "memory");
}

// Buffer descriptor of `bytes` at p (both wave-uniform).
__device__ __forceinline__ u32x4 buffer_of(const char* p, uint32_t bytes) {
    const uint64_t a = (uint64_t)(uintptr_t)p;
    return u32x4{(uint32_t)__builtin_amdgcn_readfirstlane((uint32_t)a),
                 (uint32_t)__builtin_amdgcn_readfirstlane((uint32_t)(a >> 32)) & 0xffffu,
                 (uint32_t)__builtin_amdgcn_readfirstlane(bytes), 0x00020000u};
}

// One operand: R rows of a tile (R = BM or BN), KT of the contraction, in LDS.
//
// Along the contraction (T = false) an LDS row is a row's 128 bytes, 16-byte
// chunk c of row r at slot c ^ (r / 2 % 8): 16 consecutive rows read at one
// chunk are conflict-free.  Across it (T = true) an LDS row is one k of all R
// rows, 64-byte unit u of it at u ^ (k % 4) (two units a row: u ^ (k / 2 %
// 2)), so that the four k of a transposing read lie on different banks.
template <int R, bool T>
struct Operand {
    static constexpr int BYTES = R * KT * 2;
    static constexpr int PIECES = R / (8 * WAVES);  // 1 KB loads per wavefront and k-tile
    static constexpr int RB = R / 32;               // 32-row blocks
    const char* base;
    int64_t step, left;  // bytes to the next k-tile; bytes from base to the operand's end
    uint32_t voff[PIECES];
    uint32_t most;       // bytes that a k-tile may reach from base

    static __device__ __forceinline__ int swizzle(int k) { return R == 64 ? (k >> 1) & 1 : k & 3; }

    // Rows row0 .. of `rows`; row_of(r) is tile row r's row (T = false: any, T
    // = true: row0 + r, R of them in a run).
    template <typename RowOf>
    __device__ __forceinline__ void init(const bf16* p, int64_t ld, int64_t rows, int64_t row0, int64_t K, RowOf row_of) {
        const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
        if constexpr (T) {
            base = (const char*)(p + row0);
            step = KT * ld * 2;
            left = (K * ld - row0) * 2;
            most = (uint32_t)step;
            constexpr int CH = R / 8, PER = 64 / CH;  // chunks of an LDS row, rows of a piece
#pragma unroll
            for (int q = 0; q < PIECES; ++q) {
                const int k = PER * (wave + WAVES * q) + lane / CH, ch = lane % CH;
                voff[q] = (uint32_t)(k * ld * 2) + 16 * ((((ch >> 2) ^ swizzle(k)) << 2) | (ch & 3));
            }
        } else {
            base = (const char*)(p + row0 * ld);
            step = KT * 2;
            left = (rows - row0) * ld * 2;
            most = 0xffffffffu;
#pragma unroll
            for (int q = 0; q < PIECES; ++q) {
                const int r = 8 * (wave + WAVES * q) + (lane >> 3);
                voff[q] = (uint32_t)(row_of(r) * ld * 2) + 16 * ((lane & 7) ^ ((r >> 1) & 7));
            }
        }
    }

    __device__ __forceinline__ u32x4 buffer() const {
        return buffer_of(base, (uint32_t)(left < (int64_t)most ? left : (int64_t)most));
    }
    __device__ __forceinline__ void advance() {
        base += step;
        left -= step;
    }
    __device__ __forceinline__ void load(u32x4 buf, int q, uint32_t lds) const {
        dma16(buf, voff[q], lds + ((threadIdx.x >> 6) + WAVES * q) * 1024);
    }
};

// A lane's view of an operand in LDS: row block b, k-step s (16 of KT).  The
// MFMA takes row lane % 32 and contraction 8 (lane / 32) .. + 7 of the step.
template <int R, bool T>
struct View {
    uint32_t at;
    __device__ __forceinline__ explicit View(uint32_t lds, int row0) {
        const int lane = threadIdx.x & 63;
        if constexpr (T) {
            // 16 lanes of a transposing read: 4 k x 16 rows, four rows a lane
            const int g = lane >> 4, i = lane & 15;
            const int k = 8 * (g >> 1) + (i >> 2);
            at = lds + k * (R * 2) + ((((uint32_t)row0 >> 5) ^ Operand<R, T>::swizzle(k)) << 6) + 32 * (g & 1) + 8 * (i & 3);
        } else {
            const int r = row0 + (lane & 31);
            at = lds + r * 128 + (((lane >> 5) ^ ((r >> 1) & 7)) << 4);
        }
    }
    __device__ __forceinline__ bf16x8 read(uint32_t slot, int s, int b) const {
        if constexpr (T) {
            const uint32_t a = (at ^ (b << 6)) + slot + s * (16 * R * 2);
            const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((s16x4_lds)(uintptr_t)a);
            const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((s16x4_lds)(uintptr_t)(a + 4 * R * 2));
            typedef short s16x8 __attribute__((ext_vector_type(8)));
            const s16x8 v = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
            return __builtin_bit_cast(bf16x8, v);
        } else {
            return *(const __attribute__((address_space(3))) bf16x8*)(uintptr_t)((at ^ (s << 5)) + slot + b * (32 * 128));
        }
    }
};

// The tile `tile` of product p.
template <int BM, int BN, int WM, bool XT, bool WT, int EPI>
__device__ __forceinline__ void product_tile(const FfProduct& p, int tile, char* lds) {
    constexpr int WN = WAVES / WM;
    constexpr int TM = BM / WM, TN = BN / WN;  // X and W rows of a wavefront
    constexpr int MB = TM / 32, NB = TN / 32;  // its 32 x 32 blocks
    constexpr int STAGE = (BM + BN) * KT * 2;
    constexpr int BNO = EPI == FF_GATE ? BN / 2 : BN;  // outputs of a tile
    static_assert(EPI != FF_GATE || TN % 64 == 0, "value and gate in one wavefront");
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = wave % WM, wn = wave / WM;
    const int n_tiles = (p.N + BNO - 1) / BNO;
    const int m0 = tile / n_tiles * BM, n0 = tile % n_tiles * BNO;

    Operand<BM, XT> x;
    Operand<BN, WT> w;
    x.init(p.x, p.ldx, p.M, m0, p.K, [](int r) { return (int64_t)r; });
    if constexpr (EPI == FF_GATE)  // of every 64 rows 32 are values, 32 their gates
        w.init(p.w, p.ldw, 2 * (int64_t)p.N, n0, p.K,
               [&](int r) { return (int64_t)(32 * (r >> 6) + (r & 31)) + ((r & 32) ? p.N : 0); });
    else
        w.init(p.w, p.ldw, p.N, n0, p.K, [](int r) { return (int64_t)r; });
    const uint32_t lds0 = __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)(lptr)lds);
    const View<BM, XT> xv(lds0, wm * TM);
    const View<BN, WT> wv(lds0 + BM * KT * 2, wn * TN);

    f32x16 acc[NB][MB];
#pragma unroll
    for (int i = 0; i < NB; ++i)
#pragma unroll
        for (int j = 0; j < MB; ++j)
#pragma unroll
            for (int e = 0; e < 16; ++e) acc[i][j][e] = 0.f;
    struct Ops {
        bf16x8 x[MB], w[NB];
    };
    Ops o[2];
#pragma unroll
    for (int j = 0; j < MB; ++j) o[1].x[j] = bf16x8{};
#pragma unroll
    for (int i = 0; i < NB; ++i) o[1].w[i] = bf16x8{};

    constexpr int PX = decltype(x)::PIECES, PW = decltype(w)::PIECES;
    const int nkt = (p.K + KT - 1) / KT;
    {
        const u32x4 xb = x.buffer(), wb = w.buffer();
#pragma unroll
        for (int q = 0; q < PX; ++q) x.load(xb, q, lds0);
#pragma unroll
        for (int q = 0; q < PW; ++q) w.load(wb, q, lds0 + BM * KT * 2);
    }
    // The k-tiles alternate between two stages.  A step's operands are read
    // behind the products of the step before, a tile's first ones behind the
    // last of the tile before it (the first tile's are products with zeros);
    // the next tile's loads are spread over the steps.
    uint32_t slot = 0;
    for (int t = 0; t < nkt; ++t) {
        __builtin_amdgcn_s_waitcnt(0x0070);  // vmcnt(0) lgkmcnt(0): the tile has landed, the one before has been read
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        x.advance();
        w.advance();
        const bool more = t + 1 < nkt;
        const u32x4 xb = x.buffer(), wb = w.buffer();
        const uint32_t next = lds0 + (slot ^ STAGE);
#pragma unroll
        for (int s = 0; s < 4; ++s) {
            Ops& in = o[s & 1];
            const Ops& use = o[(s & 1) ^ 1];
#pragma unroll
            for (int i = 0; i < NB; ++i) {  // a row of blocks between the reads and loads
#pragma unroll
                for (int j = 0; j < MB; ++j)
                    if (j * NB / MB == i) in.x[j] = xv.read(slot, s, j);
                in.w[i] = wv.read(slot, s, i);
                if (more) {
#pragma unroll
                    for (int q = 0; q < PX + PW; ++q)
                        if (q * 4 * NB / (PX + PW) == s * NB + i) {
                            if (q < PX)
                                x.load(xb, q, next);
                            else
                                w.load(wb, q - PX, next + BM * KT * 2);
                        }
                }
#pragma unroll
                for (int j = 0; j < MB; ++j) acc[i][j] = mfma32x32x16(use.w[i], use.x[j], acc[i][j]);
                __builtin_amdgcn_sched_barrier(0);
            }
        }
        slot ^= STAGE;
    }
#pragma unroll
    for (int i = 0; i < NB; ++i)
#pragma unroll
        for (int j = 0; j < MB; ++j) acc[i][j] = mfma32x32x16(o[1].w[i], o[1].x[j], acc[i][j]);

    // acc[i][j][e]: W row 32 i + 8 (e / 4) + 4 (lane / 32) + e % 4 of the
    // wavefront, X row 32 j + lane % 32.  The sums go through LDS, 32 X rows
    // of the wavefront at a time, so that a lane then has eight consecutive
    // outputs of a row: loads and stores run along the rows, and a lane's
    // columns are the same in every pass.
    constexpr int LDF = TN + 4;  // floats per row: 16 rows written at one column on distinct banks
    static_assert(WAVES * 32 * LDF * 4 <= 2 * STAGE, "a slab of every wavefront fits the stages");
    constexpr int TNO = EPI == FF_GATE ? TN / 2 : TN;  // outputs of a wavefront's row
    constexpr int C8 = TNO / 8, RPP = 64 / C8, PASSES = 32 / RPP;
    float* tab = (float*)lds + wave * 32 * LDF;
    const int c = 8 * (lane % C8), r0 = lane / C8;
    const int n = n0 + wn * TNO + c;
    const bool inside = n < p.N;
    // FF_GATE: the column of output c's value in the slab; its gate lies 32 on
    const int col = EPI == FF_GATE ? 64 * (c >> 5) + (c & 31) : c;
    float b0[8], b1[8], s0[8], s1[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) b0[e] = b1[e] = s0[e] = s1[e] = 0.f;
    if (EPI != FF_GATE_GRAD && p.bias != nullptr && inside) {
        load8(p.bias + n, b0);
        if constexpr (EPI == FF_GATE) load8(p.bias + p.N + n, b1);
    }
    __syncthreads();  // the stages have been read
#pragma unroll
    for (int j = 0; j < MB; ++j) {
        const int mj = m0 + wm * TM + 32 * j + r0;
        u32x2 cv[PASSES], cg[PASSES];
        int sv[PASSES], sg[PASSES];
        if constexpr (EPI == FF_GATE_GRAD) {
#pragma unroll
            for (int ps = 0; ps < PASSES; ++ps) {
                const int m = mj + RPP * ps;
                if (m >= p.M || !inside) continue;
                const int64_t at = (int64_t)m * 2 * p.N + n;
                cv[ps] = *(const u32x2*)(p.codes + at);
                cg[ps] = *(const u32x2*)(p.codes + at + p.N);
                sv[ps] = p.scales[at / EIGHT_GROUP];
                sg[ps] = p.scales[(at + p.N) / EIGHT_GROUP];
            }
        }
        __builtin_amdgcn_wave_barrier();  // the slab before has been read (LDS works in order)
#pragma unroll
        for (int i = 0; i < NB; ++i)
#pragma unroll
            for (int q = 0; q < 4; ++q)
                *(f32x4*)(tab + (lane & 31) * LDF + 32 * i + 8 * q + 4 * (lane >> 5)) =
                    f32x4{acc[i][j][4 * q], acc[i][j][4 * q + 1], acc[i][j][4 * q + 2], acc[i][j][4 * q + 3]};
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (int ps = 0; ps < PASSES; ++ps) {
            const int m = mj + RPP * ps;
            float v[8];
            load8(tab + (r0 + RPP * ps) * LDF + col, v);
            if (m >= p.M || !inside) continue;  // four lanes of a group together
            if constexpr (EPI == FF_STORE) {
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] += b0[e];
                store8(p.out + (int64_t)m * p.N + n, v);
            } else if constexpr (EPI == FF_GATE) {
                float g[8];
                load8(tab + (r0 + RPP * ps) * LDF + col + 32, g);
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    v[e] += b0[e];
                    g[e] += b1[e];
                }
                if (p.codes != nullptr) {
                    const int64_t at = (int64_t)m * 2 * p.N + n;
                    int scale;
                    *(u32x2*)(p.codes + at) = to_eight_bits(v, scale);
                    if ((lane & 3) == 0) p.scales[at / EIGHT_GROUP] = (uint8_t)scale;
                    *(u32x2*)(p.codes + at + p.N) = to_eight_bits(g, scale);
                    if ((lane & 3) == 0) p.scales[(at + p.N) / EIGHT_GROUP] = (uint8_t)scale;
                }
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] *= ff_act(p.act, g[e]);
                store8(p.out + (int64_t)m * p.N + n, v);
            } else {
                float a[8], b[8], h[8];
                const float fv = eight_value(sv[ps]), fg = eight_value(sg[ps]);
                const f32x4 kv[2] = {from_e4m3(cv[ps][0]), from_e4m3(cv[ps][1])};
                const f32x4 kg[2] = {from_e4m3(cg[ps][0]), from_e4m3(cg[ps][1])};
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const float val = kv[e >> 2][e & 3] * fv;
                    float d;
                    const float y = ff_act(p.act, kg[e >> 2][e & 3] * fg, &d);
                    a[e] = v[e] * y;
                    b[e] = v[e] * val * d;
                    h[e] = val * y;
                    s0[e] += a[e];
                    s1[e] += b[e];
                }
                if (p.out != nullptr) {
                    store8(p.out + (int64_t)m * 2 * p.N + n, a);
                    store8(p.out + (int64_t)m * 2 * p.N + p.N + n, b);
                }
                if (p.h != nullptr) store8(p.h + (int64_t)m * p.N + n, h);
            }
        }
    }
    if (EPI == FF_GATE_GRAD && p.partial != nullptr) {
#pragma unroll
        for (int d = C8; d < 64; d <<= 1)
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                s0[e] += __shfl_xor(s0[e], d);
                s1[e] += __shfl_xor(s1[e], d);
            }
        if (r0 == 0 && inside) {
            float* at = p.partial + (int64_t)(m0 / TM + wm) * 2 * p.N + n;
            store8(at, s0);
            store8(at + p.N, s1);
        }
    }
}

template <int BM, int BN, int WM, bool XT, bool WT, int EPI>
__global__ __launch_bounds__(THREADS, BM * BN > 128 * 128 ? 1 : 2) void ff_product(FfProduct p) {
    __shared__ __attribute__((aligned(256))) char lds[2 * (BM + BN) * KT * 2];
    product_tile<BM, BN, WM, XT, WT, EPI>(p, blockIdx.x, lds);
}

template <int BM, int BN, int WM>
hipError_t launch(const FfProduct& p, hipStream_t s) {
    const int bno = p.epilogue == FF_GATE ? BN / 2 : BN;
    const unsigned grid = (unsigned)((int64_t)((p.M + BM - 1) / BM) * ((p.N + bno - 1) / bno));
    if (p.epilogue == FF_GATE)
        ff_product<BM, BN, WM, false, false, FF_GATE><<<grid, THREADS, 0, s>>>(p);
    else if (p.epilogue == FF_GATE_GRAD)
        ff_product<BM, BN, WM, false, true, FF_GATE_GRAD><<<grid, THREADS, 0, s>>>(p);
    else if (p.x_t)
        ff_product<BM, BN, WM, true, true, FF_STORE><<<grid, THREADS, 0, s>>>(p);
    else if (p.w_t)
        ff_product<BM, BN, WM, false, true, FF_STORE><<<grid, THREADS, 0, s>>>(p);
    else
        ff_product<BM, BN, WM, false, false, FF_STORE><<<grid, THREADS, 0, s>>>(p);
    return hipGetLastError();
}

bool big(int64_t M) { return M > 512; }

}  // namespace

int ff_partial_rows(int64_t M) { return (int)(big(M) ? (M + 255) / 256 * 2 : (M + 127) / 128 * 2); }

hipError_t launch_ff_product(const FfProduct& p, hipStream_t s) {
    return big(p.M) ? launch<256, 256, 2>(p, s) : launch<128, 128, 2>(p, s);
}

}  // namespace pcpp

// The gated feed-forward's products (see feed_forward.h): Y = X W^T with
// either operand stored along or across the contraction, on 32x32x16 bf16
// MFMAs, with the activation, its derivative and the 8-bit checkpoint in the
// epilogue.

#include "eight_bit.h"
#include "feed_forward.h"
#include "ff_act.h"
#include "kernels.h"
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

    static constexpr __device__ __forceinline__ int swizzle(int k) { return R == 64 ? (k >> 1) & 1 : k & 3; }

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

// Tile `tile` of the product's rows and outputs: groups of kGroup tiles along
// the rows, walked along the outputs.  An XCD takes a run of tiles; the 32 that
// it works on at a time are then about 8 x 4 and share their operands in its L2.
constexpr int kGroup = 8;
template <int BM, int BNO>
__device__ __forceinline__ void place(const FfProduct& p, int tile, int& m0, int& n0) {
    const int mt = (p.M + BM - 1) / BM, nt = (p.N + BNO - 1) / BNO;
    const int group = tile / (kGroup * nt), in = tile - group * kGroup * nt;
    const int rows = min(kGroup, mt - group * kGroup);
    n0 = in / rows * BNO;
    m0 = (group * kGroup + in % rows) * BM;
}

// The tile of workgroup b: workgroups are dealt round-robin over the XCDs, an
// XCD's tiles are a run of p.per_xcd (the last may have fewer).
__device__ __forceinline__ int tile_of(const FfProduct& p, int b) {
    const int xcd = b % p.n_xcd, j = b / p.n_xcd;
    const int tile = xcd * p.per_xcd + j;
    return tile < p.tiles ? tile : -1;
}

// The outputs of a tile from its wavefronts' sums (BM / WM x BN / WN each).
template <int BM, int BN, int WM, int EPI, int ACT>
__device__ __forceinline__ void store_tile(const FfProduct& p, f32x16 (&acc)[BN * WM / (32 * WAVES)][BM / (32 * WM)], int m0,
                                           int n0, char* lds) {
    constexpr int WN = WAVES / WM;
    constexpr int TM = BM / WM, TN = BN / WN;
    constexpr int MB = TM / 32, NB = TN / 32;
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = wave % WM, wn = wave / WM;
    // acc[i][j][e]: W row 32 i + 8 (e / 4) + 4 (lane / 32) + e % 4 of the
    // wavefront, X row 32 j + lane % 32.  The sums go through LDS, 32 X rows
    // of the wavefront at a time, so that a lane then has eight consecutive
    // outputs of a row: loads and stores run along the rows, and a lane's
    // columns are the same in every pass.
    constexpr int LDF = TN + 4;  // floats per row: 16 rows written at one column on distinct banks
    static_assert(WAVES * 32 * LDF * 4 <= 2 * (BM + BN) * KT * 2, "a slab of every wavefront fits the stages");
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
                for (int e = 0; e < 8; ++e) v[e] *= ff_act<ACT>(g[e]);
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
                    const float y = ff_act<ACT>(kg[e >> 2][e & 3] * fg, &d);
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

// The tile `tile` of product p.
template <int BM, int BN, int WM, bool XT, bool WT, int EPI, int ACT>
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
    int m0, n0;
    place<BM, BNO>(p, tile, m0, n0);

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
                        if (q * 2 * NB / (PX + PW) == s * NB + i) {
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

    store_tile<BM, BN, WM, EPI, ACT>(p, acc, m0, n0, lds);
}

// One operand of the 256 x 256 tiles: the same layouts in units of 128 rows x
// KT, half of every wavefront's 128 rows (or columns) in each: unit row r is
// tile row 128 (r / 64) + r % 64, the second half's 64 rows further on.
template <bool T>
struct HalfOperand {
    static constexpr int PIECES = 4;  // 1 KB loads per wavefront and unit
    const char* base[2];          // the halves of the k-tile to load next
    int64_t step;                 // bytes to the next k-tile
    uint32_t bytes[2], last[2];   // from base to where a load may reach; T: in the last k-tile
    uint32_t less;                // T = false: what bytes shrinks by per k-tile
    int32_t tiles;                // k-tiles that are left
    uint32_t voff[PIECES];

    // row_of as in Operand, half_rows: the rows between a unit and the next.
    template <typename RowOf>
    __device__ __forceinline__ void init(const bf16* p, int64_t ld, int64_t rows, int64_t row0, int32_t K, int half_rows,
                                         int wave, RowOf row_of) {
        const int lane = threadIdx.x & 63;
        tiles = (K + KT - 1) / KT;
        if constexpr (T) {
            const int64_t half = half_rows * 2;
            base[0] = (const char*)(p + row0);
            base[1] = base[0] + half;
            step = KT * ld * 2;
            const int64_t end = (K - (int64_t)KT * (tiles - 1)) * ld * 2 - row0 * 2;
            last[0] = (uint32_t)end;
            last[1] = (uint32_t)(end > half ? end - half : 0);
            bytes[0] = tiles == 1 ? last[0] : (uint32_t)(step - row0 * 2);
            bytes[1] = tiles == 1 ? last[1] : (uint32_t)(step - row0 * 2 - half);
#pragma unroll
            for (int q = 0; q < PIECES; ++q) {
                const int k = 4 * (wave + WAVES * q) + (lane >> 4), ch = lane & 15;
                const int c = 32 * ((ch >> 2) ^ Operand<128, true>::swizzle(k)) + 8 * (ch & 3);
                voff[q] = (uint32_t)(k * ld * 2) + 2 * (128 * (c >> 6) + (c & 63));
            }
        } else {
            const int64_t left = (rows - row0) * ld * 2, half = half_rows * ld * 2;
            base[0] = (const char*)(p + row0 * ld);
            base[1] = base[0] + half;
            step = KT * 2;
            bytes[0] = (uint32_t)(left < 0xffffffffll ? left : 0xffffffffll);
            bytes[1] = (uint32_t)(left - half < 0xffffffffll ? (left > half ? left - half : 0) : 0xffffffffll);
            less = bytes[1] ? KT * 2 : 0;  // bytes[0] > 0; a row is at least K long
#pragma unroll
            for (int q = 0; q < PIECES; ++q) {
                const int r = 8 * (wave + WAVES * q) + (lane >> 3);
                voff[q] = (uint32_t)(row_of(128 * (r >> 6) + (r & 63)) * ld * 2) + 16 * ((lane & 7) ^ ((r >> 1) & 7));
            }
        }
    }
    __device__ __forceinline__ u32x4 buffer(int h) const { return buffer_of(base[h], bytes[h]); }
    // The next k-tile; past the last every load gives zeros.
    __device__ __forceinline__ void advance() {
        base[0] += step;
        base[1] += step;
        --tiles;
        if constexpr (T) {
            bytes[0] = tiles > 1 ? bytes[0] : last[0];
            bytes[1] = tiles > 1 ? bytes[1] : last[1];
        } else {
            bytes[0] -= KT * 2;
            bytes[1] -= less;
        }
        if (tiles <= 0) bytes[0] = bytes[1] = last[0] = last[1] = less = 0;
    }
};

// A 256 x 256 tile.  Four wavefronts of 128 x 128, one per SIMD: their sums
// fill the 256 accumulation registers, and LDS delivers 128 KB per k-tile for
// 2048 cycles of products.  What a loop over whole k-tiles in two stages is
// bound by is the wait for the next one: 64 KB take as long to arrive at 33
// bytes a clock as their products take, and the latency comes on top.  So the
// ring holds eight units of 16 KB, a k-tile being four: the first halves of X
// and W, the second halves of W and X.  A k-tile's products are four phases, a
// quarter of the tile each (X1 W1, X1 W2, X2 W2, X2 W1); each phase reads one
// unit into registers, the one whose products begin two phases on (one, for
// W2 and X2), and loads the unit six after it into the slot that the phase
// before the last has read.  Five units are always in flight, and a phase
// waits only for a load that was issued five phases (about 2500 cycles) before.
template <bool XT, bool WT, int EPI, int ACT>
__device__ __forceinline__ void product_tile_256(const FfProduct& p, int tile, char* lds) {
    constexpr int BNO = EPI == FF_GATE ? 128 : 256;  // outputs of a tile
    constexpr uint32_t UNIT = 128 * KT * 2;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = wave & 1, wn = wave >> 1;
    int m0, n0;
    place<256, BNO>(p, tile, m0, n0);

    HalfOperand<XT> x;
    HalfOperand<WT> w;
    x.init(p.x, p.ldx, p.M, m0, p.K, 64, wave, [](int r) { return (int64_t)r; });
    if constexpr (EPI == FF_GATE)  // of every 64 rows 32 are values, 32 their gates
        w.init(p.w, p.ldw, 2 * (int64_t)p.N, n0, p.K, 32, wave,
               [&](int r) { return (int64_t)(32 * (r >> 6) + (r & 31)) + ((r & 32) ? p.N : 0); });
    else
        w.init(p.w, p.ldw, p.N, n0, p.K, 64, wave, [](int r) { return (int64_t)r; });
    const uint32_t lds0 = __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)(lptr)lds);
    const View<128, XT> xv(lds0, 64 * wm);
    const View<128, WT> wv(lds0, 64 * wn);
    const int nkt = (p.K + KT - 1) / KT;

    f32x16 acc[4][4];
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int e = 0; e < 16; ++e) acc[i][j][e] = 0.f;

    const uint32_t dst = lds0 + wave * 1024;
    auto load = [&](const u32x4& buf, const uint32_t (&voff)[4], int q, uint32_t slot) {
        dma16(buf, voff[q], dst + slot * UNIT + q * (WAVES * 1024));
    };
    // Unit u (0: X1, 1: W1, 2: W2, 3: X2) of the k-tile that x and w stand at.
    auto buffer_of_unit = [&](int u) { return u == 0 || u == 3 ? x.buffer(u == 3) : w.buffer(u == 2); };
    auto step_after = [&](int u) {  // X2 and W2 are the last of their operand's k-tile
        if (u == 3) x.advance();
        if (u == 2) w.advance();
    };
    auto load_unit = [&](int u, uint32_t slot) {
        const u32x4 b = buffer_of_unit(u);
#pragma unroll
        for (int q = 0; q < 4; ++q)
            if (u == 0 || u == 3)
                load(b, x.voff, q, slot);
            else
                load(b, w.voff, q, slot);
        step_after(u);
    };

    struct Frag {
        bf16x8 v[2][4];  // row block, k-step
    };
    Frag xa, xb, wa, wb;
    // The phase that computes acc[ni ..][mj ..] from xr and wr, reads the unit
    // in slot `from` into `next` and loads unit `u` into slot `to`.
    auto phase = [&](const Frag& wr, const Frag& xr, int ni, int mj, Frag& next, bool next_x, uint32_t from, int u,
                     uint32_t to) {
        // This wavefront's part of the unit to read has landed (20 younger
        // loads may be in flight), and it has read the unit of two phases ago
        // (eight younger reads may be in flight); then everyone's.
        asm volatile("s_waitcnt vmcnt(20) lgkmcnt(8)\n\ts_barrier" ::: "memory");
        const u32x4 b = buffer_of_unit(u);
        // A product occupies the matrix unit for 32 cycles: reads after every
        // second one, loads after every fourth.
#pragma unroll
        for (int k = 0; k < 16; ++k) {
            const int s = k >> 2, i = (k >> 1) & 1, j = k & 1;
            acc[ni + i][mj + j] = mfma32x32x16(wr.v[i][s], xr.v[j][s], acc[ni + i][mj + j]);
            __builtin_amdgcn_sched_barrier(0);
            if (k % 2 == 0) {
                const int f = k / 2;
                next.v[f & 1][f >> 1] = next_x ? xv.read(from * UNIT, f >> 1, f & 1) : wv.read(from * UNIT, f >> 1, f & 1);
            } else if (k % 4 == 1) {
                if (u == 0 || u == 3)
                    load(b, x.voff, k / 4, to);
                else
                    load(b, w.voff, k / 4, to);
            }
            __builtin_amdgcn_sched_barrier(0);
        }
        step_after(u);
    };

#pragma unroll
    for (int u = 0; u < 8; ++u) load_unit(u & 3, u);
    asm volatile("s_waitcnt vmcnt(24)\n\ts_barrier" ::: "memory");
#pragma unroll
    for (int s = 0; s < 4; ++s)
#pragma unroll
        for (int r = 0; r < 2; ++r) {
            xa.v[r][s] = xv.read(0, s, r);
            wa.v[r][s] = wv.read(UNIT, s, r);
        }
    asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
    // Two k-tiles a round, so that every slot is a constant; W1 of the second
    // is read into W2's registers of the first and the other way round.  (An
    // odd last k-tile runs with one of zeros: leaving the round in its middle
    // made the compiler spill.)
    for (int t = 0; t < nkt; t += 2) {
        phase(wa, xa, 0, 0, wb, false, 2, 0, 0);
        phase(wb, xa, 2, 0, xb, true, 3, 1, 1);
        phase(wb, xb, 2, 2, xa, true, 4, 2, 2);
        phase(wa, xb, 0, 2, wb, false, 5, 3, 3);
        phase(wb, xa, 0, 0, wa, false, 6, 0, 4);
        phase(wa, xa, 2, 0, xb, true, 7, 1, 5);
        phase(wa, xb, 2, 2, xa, true, 0, 2, 6);
        phase(wb, xb, 0, 2, wa, false, 1, 3, 7);
    }
    // Loads past the end are still on their way (zeros) to the slots.
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    store_tile<256, 256, 2, EPI, ACT>(p, acc, m0, n0, lds);
}

template <int BM, int BN, int WM, bool XT, bool WT, int EPI, int ACT>
__global__ __launch_bounds__(THREADS, BM * BN > 128 * 128 ? 1 : 2) void ff_product(FfProduct p) {
    __shared__ __attribute__((aligned(256))) char lds[2 * (BM + BN) * KT * 2];
    const int tile = tile_of(p, blockIdx.x);
    if (tile < 0) return;
    if constexpr (BM == 256)
        product_tile_256<XT, WT, EPI, ACT>(p, tile, lds);
    else
        product_tile<BM, BN, WM, XT, WT, EPI, ACT>(p, tile, lds);
}

// Up to three products of FF_STORE in one launch: first those with both
// operands across the contraction (the weights' gradients, the longest), then
// one with W alone across it.  Their tiles together leave fewer compute units
// idle at the end than three launches do.
struct FfGroup {
    FfProduct p[3];
    int32_t n;
};
template <int BM, int BN, int WM>
__global__ __launch_bounds__(THREADS, BM * BN > 128 * 128 ? 1 : 2) void ff_products(FfGroup g) {
    __shared__ __attribute__((aligned(256))) char lds[2 * (BM + BN) * KT * 2];
    const int xcd = blockIdx.x % g.p[0].n_xcd;
    int j = blockIdx.x / g.p[0].n_xcd, which = 0;
    while (which < g.n - 1 && j >= g.p[which].per_xcd) j -= g.p[which++].per_xcd;
    const FfProduct& p = g.p[which];
    const int tile = xcd * p.per_xcd + j;
    if (tile >= p.tiles) return;
    if (p.x_t) {
        if constexpr (BM == 256)
            product_tile_256<true, true, FF_STORE, 0>(p, tile, lds);
        else
            product_tile<BM, BN, WM, true, true, FF_STORE, 0>(p, tile, lds);
    } else {
        if constexpr (BM == 256)
            product_tile_256<false, true, FF_STORE, 0>(p, tile, lds);
        else
            product_tile<BM, BN, WM, false, true, FF_STORE, 0>(p, tile, lds);
    }
}

// The tiles of p, dealt over the XCDs.
void set_tiles(FfProduct& p, int bm, int bno) {
    const int cus = device_cus();
    p.tiles = (p.M + bm - 1) / bm * ((p.N + bno - 1) / bno);
    p.n_xcd = layout_for(cus, cus).n_xcd;
    p.per_xcd = (p.tiles + p.n_xcd - 1) / p.n_xcd;
}

template <int BM, int BN, int WM>
hipError_t launch(FfProduct p, hipStream_t s) {
    set_tiles(p, BM, p.epilogue == FF_GATE ? BN / 2 : BN);
    const unsigned grid = (unsigned)p.n_xcd * p.per_xcd;
    const bool silu = p.act == PCPP_ACT_SILU;
    auto run = [&](auto kernel) { kernel<<<grid, THREADS, 0, s>>>(p); };
    if (p.epilogue == FF_GATE)
        run(silu ? ff_product<BM, BN, WM, false, false, FF_GATE, PCPP_ACT_SILU>
                 : ff_product<BM, BN, WM, false, false, FF_GATE, PCPP_ACT_GELU>);
    else if (p.epilogue == FF_GATE_GRAD)
        run(silu ? ff_product<BM, BN, WM, false, true, FF_GATE_GRAD, PCPP_ACT_SILU>
                 : ff_product<BM, BN, WM, false, true, FF_GATE_GRAD, PCPP_ACT_GELU>);
    else
        run(ff_product<BM, BN, WM, false, false, FF_STORE, 0>);
    return hipGetLastError();
}

template <int BM, int BN, int WM>
hipError_t launch_group(const FfProduct* p, int n, hipStream_t s) {
    FfGroup g = {};
    g.n = n;
    unsigned grid = 0;
    for (int i = 0; i < n; ++i) {
        g.p[i] = p[i];
        set_tiles(g.p[i], BM, BN);
        grid += (unsigned)g.p[i].n_xcd * g.p[i].per_xcd;
    }
    ff_products<BM, BN, WM><<<grid, THREADS, 0, s>>>(g);
    return hipGetLastError();
}

bool big(int64_t M) { return M > 512; }

}  // namespace

int ff_partial_rows(int64_t M) { return (int)(big(M) ? (M + 255) / 256 * 2 : (M + 127) / 128 * 2); }

hipError_t launch_ff_product(const FfProduct& p, hipStream_t s) {
    return big(p.M) ? launch<256, 256, 2>(p, s) : launch<128, 128, 2>(p, s);
}

hipError_t launch_ff_products(const FfProduct* p, int n, hipStream_t s) {
    return big(p[0].M) ? launch_group<256, 256, 2>(p, n, s) : launch_group<128, 128, 2>(p, n, s);
}

}  // namespace pcpp

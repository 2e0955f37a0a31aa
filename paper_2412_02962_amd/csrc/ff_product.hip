// The gated feed-forward's products (see feed_forward.h): Y = X W^T with
// either operand stored along or across the contraction, on 32x32x16 bf16
// MFMAs, with the activation, its derivative and the 8-bit checkpoint in the
// epilogue.

#include "checkpoint.h"
#include "column_sums.h"
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

// The kinds of tile: their rows of X and W (wider with an epilogue that halves
// the outputs or whose operations cover the wait for operands), ring in LDS, and
// how many of their workgroups share a compute unit.
// TILE_64_THREE, FF_GATE_GRAD's alone, is TILE_64 with a ring of two stages.
enum { TILE_64, TILE_128, TILE_256, TILE_KINDS, TILE_64_THREE = TILE_KINDS };
constexpr bool is_64(int kind) { return kind == TILE_64 || kind == TILE_64_THREE; }
constexpr int rows_x(int kind) { return is_64(kind) ? 64 : kind == TILE_128 ? 128 : 256; }
constexpr int rows_w(int kind, int epilogue) {
    return is_64(kind) || (kind == TILE_128 && epilogue == FF_STORE) ? 128 : 256;
}
constexpr int outputs_of(int kind, int epilogue) { return rows_w(kind, epilogue) / (epilogue == FF_GATE ? 2 : 1); }
constexpr int lds_bytes(int kind) {
    return (kind == TILE_64 ? 72 : kind == TILE_128 ? 80 : kind == TILE_256 ? 128 : 48) * 1024;
}
constexpr int per_cu(int kind) { return kind == TILE_64_THREE ? 3 : kind == TILE_256 ? 1 : 2; }

typedef __attribute__((address_space(3))) void* lptr;
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) s16x4* s16x4_lds;

// 16 bytes per lane into LDS at lds + 16 lane, from byte voff of the buffer
// (zeros past its end).  Inline assembly, so that the compiler does not wait
// for loads in flight before every LDS read: the kernel orders them itself.
__device__ __forceinline__ void dma16(u32x4 buffer, uint32_t voff, uint32_t lds) {
    asm volatile("s_nop 0\n\tbuffer_load_dwordx4 %0, %1, 0 offen lds" ::"v"(voff), "s"(buffer), "{m0}"(lds) : "memory");
}

// v in a scalar register that a scalar instruction wrote.  A memory instruction
// may read one that a vector instruction wrote (readfirstlane) only five wait
// states later; the compiler keeps to that for instructions it knows, not for
// dma16's, whose buffers' words therefore all pass through here.  (Waiting the
// five states instead: 1 % more time at 32768 x 1280 x 5120.)
__device__ __forceinline__ uint32_t scalar(uint32_t v) {
    uint32_t s;
    asm("s_mov_b32 %0, %1" : "=s"(s) : "s"(__builtin_amdgcn_readfirstlane(v)));
    return s;
}

// Buffer descriptor of `bytes` at p (both wave-uniform).
__device__ __forceinline__ u32x4 buffer_of(const char* p, uint32_t bytes) {
    const uint64_t a = (uint64_t)(uintptr_t)p;
    return u32x4{scalar((uint32_t)a), scalar((uint32_t)(a >> 32) & 0xffffu), scalar(bytes), 0x00020000u};
}

// Where the k-tiles of an operand's rows are read from: what lies past the
// last row, the contraction's end or the last of the k-tiles comes as zeros.
// T: stored across the contraction, [K, rows], else [rows, K].
template <bool T>
struct Source {
    const char* base;      // the k-tile to load next
    int64_t step;          // bytes to the one after it
    uint32_t bytes, last;  // from base to where a load may reach; T: in the last k-tile
    int32_t tiles;         // k-tiles that are left

    // `count` k-tiles from k-tile `first` of rows row0 .. of p [rows, K].
    __device__ __forceinline__ void init(const bf16* p, int64_t ld, int64_t rows, int64_t row0, int32_t K, int32_t first,
                                         int32_t count) {
        tiles = count;
        if constexpr (T) {
            step = KT * ld * 2;
            base = (const char*)(p + row0) + first * step;
            const int64_t full = step - row0 * 2, end = (K - (int64_t)KT * (first + count - 1)) * ld * 2 - row0 * 2;
            last = (uint32_t)(end < full ? end : full);
            bytes = count == 1 ? last : (uint32_t)full;
        } else {
            step = KT * 2;
            base = (const char*)(p + row0 * ld) + first * step;
            const int64_t left = (rows - row0) * ld * 2 - first * step;
            bytes = (uint32_t)(left < 0xffffffffll ? left : 0xffffffffll);
        }
    }
    // From `off` bytes further on.
    __device__ __forceinline__ u32x4 buffer(uint32_t off) const {
        return buffer_of(base + off, bytes > off ? bytes - off : 0);
    }
    __device__ __forceinline__ void advance() {
        base += step;
        --tiles;
        if constexpr (T)
            bytes = tiles > 1 ? bytes : last;
        else
            bytes -= KT * 2;
        if (tiles <= 0) bytes = 0;
    }
};

// R rows of a k-tile in LDS, and what a wavefront loads of them: PIECES loads
// of 1 KB.
//
// Along the contraction (T = false) an LDS row is a row's 128 bytes, 16-byte
// chunk c of row r at slot c ^ (r / 2 % 8): 16 consecutive rows read at one
// chunk are conflict-free.  Across it (T = true) an LDS row is one k of all R
// rows, 64-byte unit u of it at u ^ swizzle(k), so that the four k of a
// transposing read lie on different banks.
template <int R, bool T>
struct Layout {
    static constexpr int BYTES = R * KT * 2;
    static constexpr int PIECES = R / (8 * WAVES);
    static constexpr __device__ __forceinline__ int swizzle(int k) { return R == 64 ? (k >> 1) & 1 : k & 3; }

    // The byte of a k-tile that this lane reads in the wavefront's q-th load;
    // row_of(r): LDS row r's row (T: r, whole 128-byte lines of a k).
    template <typename RowOf>
    static __device__ __forceinline__ uint32_t offset(int q, int wave, int64_t ld, RowOf row_of) {
        const int lane = threadIdx.x & 63;
        if constexpr (T) {
            constexpr int CH = R / 8, PER = 64 / CH;  // chunks of an LDS row, rows of a load
            const int k = PER * (wave + WAVES * q) + lane / CH, ch = lane % CH;
            return (uint32_t)(k * ld * 2) + 64 * ((ch >> 2) ^ swizzle(k)) + 16 * (ch & 3);
        } else {
            const int r = 8 * (wave + WAVES * q) + (lane >> 3);
            return (uint32_t)(row_of(r) * ld * 2) + 16 * ((lane & 7) ^ ((r >> 1) & 7));
        }
    }
};

// The 32 rows of a tile that are block b of the w-th of its wavefronts along
// them: a run of its own rows, or, where the operand lies across the
// contraction, 32 of every 64 (so that 64 neighbouring rows, a 128-byte line of
// a k, are read together).
template <bool T>
constexpr __device__ __forceinline__ int block_row(int b, int w, int run) {
    return T ? 64 * b + 32 * w : run * w + 32 * b;
}

// A lane's view of an operand in LDS: the wavefront's row block b, k-step s (16
// of KT).  The MFMA takes row lane % 32 and contraction 8 (lane / 32) .. + 7 of
// the step.
template <int R, bool T>
struct View {
    uint32_t at;
    __device__ __forceinline__ explicit View(uint32_t lds, int row0) {
        const int lane = threadIdx.x & 63;
        if constexpr (T) {
            // 16 lanes of a transposing read: 4 k x 16 rows, four rows a lane
            const int g = lane >> 4, i = lane & 15;
            const int k = 8 * (g >> 1) + (i >> 2);
            at = lds + k * (R * 2) + ((((uint32_t)row0 >> 5) ^ Layout<R, T>::swizzle(k)) << 6) + 32 * (g & 1) + 8 * (i & 3);
        } else {
            const int r = row0 + (lane & 31);
            at = lds + r * 128 + (((lane >> 5) ^ ((r >> 1) & 7)) << 4);
        }
    }
    __device__ __forceinline__ bf16x8 read(uint32_t slot, int s, int b) const {
        if constexpr (T) {
            const uint32_t a = (at ^ (b << 7)) + slot + s * (16 * R * 2);
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

// An item of a product's work: a tile of its rows and outputs, and a run of
// its k-tiles.  Workgroups are dealt round-robin over the XCDs; an XCD takes a
// run of items, and those are ordered as pieces of the contraction, then
// groups of kGroup tiles along the rows, walked along the outputs: what an XCD
// works on at a time is about square and shares its operands in the L2.
constexpr int kGroup = 4;
struct Item {
    int m0, n0, piece, first, count;  // rows and outputs from; piece; its k-tiles
};
template <int BM, int BNO>
__device__ __forceinline__ Item item_of(const FfProduct& p, int item) {
    const int mt = (p.M + BM - 1) / BM, nt = (p.N + BNO - 1) / BNO;
    Item it;
    it.piece = item / (mt * nt);
    const int tile = item - it.piece * mt * nt;
    const int group = tile / (kGroup * nt), in = tile - group * kGroup * nt;
    const int rows = min(kGroup, mt - group * kGroup);
    it.n0 = in / rows * BNO;
    it.m0 = (group * kGroup + in % rows) * BM;
    const int nkt = (p.K + KT - 1) / KT;
    it.first = (int)((int64_t)nkt * it.piece / p.pieces);
    it.count = (int)((int64_t)nkt * (it.piece + 1) / p.pieces) - it.first;
    return it;
}

// The outputs of a tile from its wavefronts' sums: two wavefronts along X's
// rows, two along W's.
template <int KIND, bool XT, bool WT, int EPI, int ACT>
__device__ __forceinline__ void store_tile(const FfProduct& p, const Item& it,
                                           f32x16 (&acc)[rows_w(KIND, EPI) / 64][rows_x(KIND) / 64], char* lds) {
    const int m0 = it.m0, n0 = it.n0;
    constexpr int TM = rows_x(KIND) / 2, TN = rows_w(KIND, EPI) / 2;  // of a wavefront
    constexpr int NB = TN / 32;
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = wave & 1, wn = wave >> 1;
    // acc[i][j][e]: W row 32 i + 8 (e / 4) + 4 (lane / 32) + e % 4 of the
    // wavefront, X row 32 j + lane % 32.  The sums go through LDS, 32 X rows
    // of the wavefront at a time, so that a lane then has eight consecutive
    // outputs of a row: loads and stores run along the rows, and a lane's
    // columns are the same in every pass.
    constexpr int LDF = TN + 4;  // floats per row: 16 rows written at one column on distinct banks
    static_assert(WAVES * 32 * LDF * 4 <= lds_bytes(KIND), "a slab of every wavefront fits the stages");
    constexpr int TNO = EPI == FF_GATE ? TN / 2 : TN;  // outputs of a wavefront's row
    constexpr int C8 = TNO / 8, RPP = 64 / C8, PASSES = 32 / RPP;
    float* tab = (float*)lds + wave * 32 * LDF;
    const int c = 8 * (lane % C8), r0 = lane / C8;
    const int n = n0 + (EPI == FF_GATE ? wn * TNO + c : block_row<WT>(c >> 5, wn, TN) + (c & 31));
    const bool inside = n < p.N;
    // FF_GATE: the column of output c's value in the slab; its gate lies 32 on
    const int col = EPI == FF_GATE ? 64 * (c >> 5) + (c & 31) : c;
    float b0[8], b1[8], s0[8], s1[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) b0[e] = b1[e] = s0[e] = s1[e] = 0.f;
    const bool whole = EPI != FF_STORE || p.pieces == 1;
    if (EPI != FF_GATE_GRAD && whole && p.bias != nullptr && inside) {
        load8(p.bias + n, b0);
        if constexpr (EPI == FF_GATE) load8(p.bias + p.N + n, b1);
    }
    __syncthreads();  // the stages have been read
#pragma unroll
    for (int j = 0; j < TM / 32; ++j) {
        const int mj = m0 + block_row<XT>(j, wm, TM) + r0;
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
                if (!whole) {
                    store8(p.part + ((int64_t)it.piece * p.M + m) * p.N + n, v);
                    continue;
                }
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

// A 64 x 128 tile, for few tiles: four wavefronts of 32 x 64 and a ring of
// three stages of 24 KB, two workgroups to a compute unit (six stages and one
// workgroup were no faster alone, 0.3 us a k-tile, about what 24 KB take from
// the L2, and left the epilogue uncovered: the up product of 2093 x 640 x 2560
// 45 us, now 31).  A step's operands are read behind the products of the step
// before, a k-tile's first ones behind the last of the one before it (the
// first k-tile's are products with zeros).
//
// Two stages and three workgroups cover more of the epilogues and less of the
// loads: the gate's gradient takes them where there are tiles for all three.
// 2093 x 640 x 2560 (660 tiles) 25.5 -> 22.9 us; with fewer, a training step of
// 1024 x 640 x 2560 (320 tiles) 84.2 -> 85.0, of 77 x 2048 x 5504 92 -> 99.
template <int KIND, bool XT, bool WT, int EPI, int ACT>
__device__ __forceinline__ void product_tile_64x128(const FfProduct& p, int item, char* lds) {
    constexpr int STAGE = (64 + 128) * KT * 2, STAGES = lds_bytes(KIND) / STAGE;
    typedef Layout<64, XT> LX;
    typedef Layout<128, WT> LW;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = wave & 1, wn = wave >> 1;
    const Item it = item_of<64, outputs_of(KIND, EPI)>(p, item);

    Source<XT> x;
    Source<WT> w;
    x.init(p.x, p.ldx, p.M, it.m0, p.K, it.first, it.count);
    w.init(p.w, p.ldw, EPI == FF_GATE ? 2 * (int64_t)p.N : p.N, it.n0, p.K, it.first, it.count);
    uint32_t xoff[LX::PIECES], woff[LW::PIECES];
#pragma unroll
    for (int q = 0; q < LX::PIECES; ++q) xoff[q] = LX::offset(q, wave, p.ldx, [](int r) { return (int64_t)r; });
#pragma unroll
    for (int q = 0; q < LW::PIECES; ++q)  // FF_GATE: of every 64 rows 32 are values, 32 their gates
        woff[q] = LW::offset(q, wave, p.ldw, [&](int r) {
            return EPI == FF_GATE ? (int64_t)(32 * (r >> 6) + (r & 31)) + ((r & 32) ? p.N : 0) : (int64_t)r;
        });
    const uint32_t lds0 = __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)(lptr)lds);
    const View<64, XT> xv(lds0, 32 * wm);
    const View<128, WT> wv(lds0 + LX::BYTES, block_row<WT>(0, wn, 64));

    f32x16 acc[2][1];
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int e = 0; e < 16; ++e) acc[i][0][e] = 0.f;
    struct Ops {
        bf16x8 x, w[2];
    };
    Ops o[2];
    o[1].x = o[1].w[0] = o[1].w[1] = bf16x8{};

    uint32_t rd = 0, wr = 0;
    auto next_of = [](uint32_t s) { return s + STAGE == STAGES * STAGE ? 0 : s + STAGE; };
    auto load_x = [&](int q, const u32x4& b) { dma16(b, xoff[q], lds0 + wr + (wave + WAVES * q) * 1024); };
    auto load_w = [&](int q, const u32x4& b) { dma16(b, woff[q], lds0 + wr + LX::BYTES + (wave + WAVES * q) * 1024); };
#pragma unroll
    for (int t = 0; t < STAGES - 1; ++t) {
        const u32x4 xb = x.buffer(0), wb = w.buffer(0);
#pragma unroll
        for (int q = 0; q < LX::PIECES; ++q) load_x(q, xb);
#pragma unroll
        for (int q = 0; q < LW::PIECES; ++q) load_w(q, wb);
        x.advance();
        w.advance();
        wr = next_of(wr);
    }
    static_assert(LX::PIECES + LW::PIECES == 6, "six of a wavefront's loads are a k-tile's");
    for (int t = 0; t < it.count; ++t) {
        // The k-tile has landed and the one before has been read, everyone's.
        asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(6 * (STAGES - 2)) : "memory");
        const u32x4 xb = x.buffer(0), wb = w.buffer(0);
#pragma unroll
        for (int s = 0; s < 4; ++s) {
            Ops& in = o[s & 1];
            const Ops& use = o[(s & 1) ^ 1];
            in.x = xv.read(rd, s, 0);
#pragma unroll
            for (int i = 0; i < 2; ++i) in.w[i] = wv.read(rd, s, i);
            if (s < LX::PIECES) load_x(s, xb);
            load_w(s, wb);
#pragma unroll
            for (int i = 0; i < 2; ++i) acc[i][0] = mfma32x32x16(use.w[i], use.x, acc[i][0]);
            __builtin_amdgcn_sched_barrier(0);
        }
        x.advance();
        w.advance();
        rd = next_of(rd);
        wr = next_of(wr);
    }
#pragma unroll
    for (int i = 0; i < 2; ++i) acc[i][0] = mfma32x32x16(o[1].w[i], o[1].x, acc[i][0]);
    // Loads past the end are still on their way (zeros) to the stages.
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    store_tile<KIND, XT, WT, EPI, ACT>(p, it, acc, lds);
}

// A 128 x 256 tile (FF_STORE: 128 x 128), two workgroups to a compute unit:
// while one waits at a barrier or for LDS, or is in its epilogue (an
// exponential, a reciprocal and some 20 operations an output, and up to 8 bytes
// of memory traffic), the other's products run.  Four wavefronts of 64 x 128
// (64 x 64), two per SIMD.
//
// A loop over whole k-tiles in two stages waits for the next one: its bytes
// take as long to arrive as its products take, and the latency comes on top.
// So the ring holds ten units of 8 KB, a k-tile being six (four) in the order
// W0 X0 X1 W1 .., and a phase is the products of one of the W units with both
// of X.  The last phase reads the next k-tile's W0 and X0 into registers, phase
// 0 X1 (used by its second half) and W1, the others one W unit each; a phase
// loads into the slots that the phase before the last has read.  Four to six
// units of a workgroup are always in flight.
//
// The up product of 32768 x 1280 x 5120 (859 GF): 780 to 980 us, 1.30 M cycles
// at the 1.4 to 1.5 GHz that the power limit leaves, MFMA busy in 63 % of them
// (one workgroup to a compute unit: 1.98 M, 41 %); with its checkpoint, 16385
// tokens, 430 to 495 us.  The gate's gradient there: 335 to 380 us, 34 %, of
// which about 100 are its 520 MB of results.
template <bool XT, bool WT, int EPI, int ACT>
__device__ __forceinline__ void product_tile_128(const FfProduct& p, int item, char* lds) {
    constexpr int TN = rows_w(TILE_128, EPI) / 2;          // W rows of a wavefront
    constexpr int NW = TN / 32, UNITS = NW + 2;            // W units, units of a k-tile
    constexpr uint32_t UNIT = 64 * KT * 2, RING = 10 * UNIT;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = wave & 1, wn = wave >> 1;
    const Item it = item_of<128, outputs_of(TILE_128, EPI)>(p, item);

    // Unit i has block i of both wavefronts along the rows; FF_GATE's W: 32
    // outputs' values for even i, their gates for odd.
    typedef Layout<64, XT> LX;
    typedef Layout<64, WT> LW;
    Source<XT> x;
    Source<WT> w;
    x.init(p.x, p.ldx, p.M, it.m0, p.K, it.first, it.count);
    w.init(p.w, p.ldw, EPI == FF_GATE ? 2 * (int64_t)p.N : p.N, it.n0, p.K, it.first, it.count);
    uint32_t xoff[2], woff[2];
#pragma unroll
    for (int q = 0; q < 2; ++q) {
        xoff[q] = LX::offset(q, wave, p.ldx,
                             [](int r) { return (int64_t)(block_row<XT>(0, r >> 5, 64) + (r & 31)); });
        woff[q] = LW::offset(q, wave, p.ldw, [](int r) {
            return (int64_t)(block_row<WT>(0, r >> 5, EPI == FF_GATE ? TN / 2 : TN) + (r & 31));
        });
    }
    const uint32_t x_off = XT ? 128 : (uint32_t)(64 * p.ldx);
    uint32_t w_off[NW];
#pragma unroll
    for (int i = 0; i < NW; ++i)
        w_off[i] = EPI == FF_GATE ? (uint32_t)((32 * (i >> 1) + (i & 1 ? (int64_t)p.N : 0)) * p.ldw * 2)
                   : WT           ? 128 * i
                                  : (uint32_t)(64 * i * p.ldw);
    const uint32_t lds0 = __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)(lptr)lds);
    const View<64, XT> xv(lds0, 32 * wm);
    const View<64, WT> wv(lds0, 32 * wn);

    f32x16 acc[NW][2];
#pragma unroll
    for (int i = 0; i < NW; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int e = 0; e < 16; ++e) acc[i][j][e] = 0.f;

    struct Frag {
        bf16x8 v[4];  // k-steps
    };
    uint32_t rd = 0, wr = 0;  // slots to read and to load next
    auto load = [&](int u, int q, const u32x4& b) {
        dma16(b, u == 1 || u == 2 ? xoff[q] : woff[q], lds0 + wave * 1024 + wr + q * (WAVES * 1024));
    };
    // Unit u in the order of a k-tile.
    auto buffer_of_unit = [&](int u) {
        return u == 1 ? x.buffer(0) : u == 2 ? x.buffer(x_off) : w.buffer(w_off[u == 0 ? 0 : u - 2]);
    };
    auto loaded = [&](int u) {
        if (u == 2) x.advance();
        if (u == UNITS - 1) w.advance();
        wr = wr + UNIT == RING ? 0 : wr + UNIT;
    };
    auto step_read = [&]() { rd = rd + UNIT == RING ? 0 : rd + UNIT; };

    constexpr int AHEAD = NW == 4 ? 9 : 8;  // units loaded before the first phase
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) {
        const u32x4 b = buffer_of_unit(u % UNITS);
        load(u % UNITS, 0, b);
        load(u % UNITS, 1, b);
        loaded(u % UNITS);
    }
    Frag wa, wb, xa, xb, xc;
    asm volatile("s_waitcnt vmcnt(%0)\n\ts_barrier" ::"n"(2 * (AHEAD - 2)) : "memory");
#pragma unroll
    for (int s = 0; s < 4; ++s) wa.v[s] = wv.read(rd, s, 0);
    step_read();
#pragma unroll
    for (int s = 0; s < 4; ++s) xa.v[s] = xv.read(rd, s, 0);
    step_read();

    // Phase i: products of wc with x0 and x1; the reads and loads listed above.
    // Before it, this wavefront's part of the units to read has landed (four to
    // six younger units, two loads each, may be in flight) and it has read
    // those of two phases ago (the phase before read two units, or one, of at
    // least four reads each); then everyone's.
    auto phase = [&](int i, const Frag& wc, Frag& wnext, const Frag& x0, Frag& x1, Frag& x0next) {
        if (NW == 2)
            asm volatile("s_waitcnt vmcnt(8) lgkmcnt(8)\n\ts_barrier" ::: "memory");
        else if (i < 2)
            asm volatile("s_waitcnt vmcnt(10) lgkmcnt(8)\n\ts_barrier" ::: "memory");
        else
            asm volatile("s_waitcnt vmcnt(12) lgkmcnt(4)\n\ts_barrier" ::: "memory");
        // the units to load: W1 | W2 W3 | W0 X0 of the k-tile after the next |
        // X1; of four units W0 X0 | X1 W1, both of the k-tile after the next
        const int u0 = NW == 2 ? 2 * i : i == 0 ? 3 : i == 1 ? 4 : i == 2 ? 0 : 2;
        const int nu = NW == 2 || i == 1 || i == 2 ? 2 : 1;
        u32x4 b = buffer_of_unit(u0);
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            // phase 0 begins with x0 alone: x1 is on its way
            const int j = i == 0 ? k >> 2 : k & 1, s = i == 0 ? k & 3 : k >> 1;
            acc[i][j] = mfma32x32x16(wc.v[s], j ? x1.v[s] : x0.v[s], acc[i][j]);
            __builtin_amdgcn_sched_barrier(0);
            if (i == 0) {
                if (k < 2) {
                    x1.v[2 * k] = xv.read(rd, 2 * k, 0);
                    x1.v[2 * k + 1] = xv.read(rd, 2 * k + 1, 0);
                    if (k == 1) step_read();
                } else if (k < 6) {
                    wnext.v[k - 2] = wv.read(rd, k - 2, 0);
                    if (k == 5) step_read();
                }
            } else if (k < 4) {
                wnext.v[k] = wv.read(rd, k, 0);
                if (k == 3) step_read();
            } else if (i == NW - 1) {
                x0next.v[k - 4] = xv.read(rd, k - 4, 0);
                if (k == 7) step_read();
            }
            if (k % 2 == 1 && (nu == 2 || k > 4)) {
                const int c = nu == 2 ? k >> 1 : (k - 5) >> 1;  // 0 .. 2 nu - 1
                if (c == 2) b = buffer_of_unit(u0 + 1);
                load(u0 + (c >> 1), c & 1, b);
                if (c & 1) loaded(u0 + (c >> 1));
            }
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    // Products before the other workgroup's epilogue; without much of one the two
    // also get different priorities, so that they do not stay in step, by the
    // wavefront's slot on its SIMD, the low bit of the hardware's id (the training
    // step of 8192 x 640 x 2560: 336 us, all equal 355; with an epilogue it costs,
    // forward 32768 x 1280 x 5120 1228, all equal 1192).
    if (EPI == FF_STORE && __builtin_amdgcn_s_getreg(4 | (3 << 11)) & 1)
        __builtin_amdgcn_s_setprio(3);
    else
        __builtin_amdgcn_s_setprio(1);
    for (int t = 0; t < it.count; t += 2) {  // an odd last k-tile runs with one of zeros
#pragma unroll
        for (int i = 0; i < NW; i += 2) {
            phase(i, wa, wb, xa, xb, xc);
            phase(i + 1, wb, wa, xa, xb, xc);
        }
#pragma unroll
        for (int i = 0; i < NW; i += 2) {
            phase(i, wa, wb, xc, xb, xa);
            phase(i + 1, wb, wa, xc, xb, xa);
        }
    }
    __builtin_amdgcn_s_setprio(0);
    // Loads past the end are still on their way (zeros) to the slots.
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    store_tile<TILE_128, XT, WT, EPI, ACT>(p, it, acc, lds);
}

// A 256 x 256 tile, for the products without an epilogue where there are tiles
// enough: half the bytes a product of the 128 x 128 tiles, one workgroup to a
// compute unit.  Four wavefronts of 128 x 128, one per SIMD, whose sums fill
// the 256 accumulation registers.  The ring holds eight units of 16 KB, a k-tile
// being four: the first halves of X and W, the second halves of W and X.  A
// k-tile's products are four phases, a quarter of the tile each (X1 W1, X1 W2,
// X2 W2, X2 W1); each phase reads one unit into registers, the one whose
// products begin two phases on (one, for W2 and X2), and loads the unit six
// after it into the slot that the phase before the last has read.  A phase
// waits only for a load that was issued five phases (about 2500 cycles) before.
//
// The down product of 32768 x 1280 x 5120 (429 GF): 365 to 435 us, 0.65 M cycles
// at 1.5 GHz, MFMA busy in 63 %; the gradients of 16385 tokens (1074 GF): 870 to
// 1000 us, 68 %, 1.7 GHz.  A k-tile takes 2700 cycles, 2480 without its loads,
// 2270 without its reads too, 2048 of MFMA.
template <bool XT, bool WT>
__device__ __forceinline__ void product_tile_256x256(const FfProduct& p, int item, char* lds) {
    constexpr uint32_t UNIT = 128 * KT * 2;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = wave & 1, wn = wave >> 1;
    const Item it = item_of<256, 256>(p, item);

    // Unit h has blocks 2 h and 2 h + 1 of both wavefronts along the rows.
    typedef Layout<128, XT> LX;
    typedef Layout<128, WT> LW;
    Source<XT> x;
    Source<WT> w;
    x.init(p.x, p.ldx, p.M, it.m0, p.K, it.first, it.count);
    w.init(p.w, p.ldw, p.N, it.n0, p.K, it.first, it.count);
    uint32_t xoff[4], woff[4];
    auto row_of = [](int r) { return (int64_t)(128 * (r >> 6) + (r & 63)); };
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        xoff[q] = LX::offset(q, wave, p.ldx, row_of);
        woff[q] = LW::offset(q, wave, p.ldw, row_of);
    }
    const uint32_t x_half = XT ? 256 : (uint32_t)(128 * p.ldx), w_half = WT ? 256 : (uint32_t)(128 * p.ldw);
    const uint32_t lds0 = __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)(lptr)lds);
    const View<128, XT> xv(lds0, block_row<XT>(0, wm, 64));
    const View<128, WT> wv(lds0, block_row<WT>(0, wn, 64));

    f32x16 acc[4][4];
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int e = 0; e < 16; ++e) acc[i][j][e] = 0.f;

    // Unit u (0: X1, 1: W1, 2: W2, 3: X2) of the k-tile that x and w stand at.
    auto buffer_of_unit = [&](int u) {
        return u == 0 || u == 3 ? x.buffer(u == 3 ? x_half : 0) : w.buffer(u == 2 ? w_half : 0);
    };
    auto load = [&](int u, int q, const u32x4& b, uint32_t slot) {
        dma16(b, u == 0 || u == 3 ? xoff[q] : woff[q], lds0 + slot * UNIT + (wave + WAVES * q) * 1024);
    };
    auto loaded = [&](int u) {  // X2 and W2 are the last of their operand's k-tile
        if (u == 3) x.advance();
        if (u == 2) w.advance();
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
                load(u, k / 4, b, to);
            }
            __builtin_amdgcn_sched_barrier(0);
        }
        loaded(u);
    };
#pragma unroll
    for (int u = 0; u < 8; ++u) {
        const u32x4 b = buffer_of_unit(u & 3);
#pragma unroll
        for (int q = 0; q < 4; ++q) load(u & 3, q, b, u);
        loaded(u & 3);
    }
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
    for (int t = 0; t < it.count; t += 2) {
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
    store_tile<TILE_256, XT, WT, FF_STORE, 0>(p, it, acc, lds);
}

template <int KIND, bool XT, bool WT, int EPI, int ACT>
__device__ __forceinline__ void product_tile(const FfProduct& p, int item, char* lds) {
    if constexpr (KIND == TILE_256)
        product_tile_256x256<XT, WT>(p, item, lds);
    else if constexpr (KIND == TILE_128)
        product_tile_128<XT, WT, EPI, ACT>(p, item, lds);
    else
        product_tile_64x128<KIND, XT, WT, EPI, ACT>(p, item, lds);
}

// FF_STORE or FF_GATE with both operands along the contraction.
template <int KIND, int EPI, int ACT>
__global__ __launch_bounds__(THREADS, per_cu(KIND)) void ff_product(FfProduct p) {
    __shared__ __attribute__((aligned(256))) char lds[lds_bytes(KIND)];
    const int item = (int)(blockIdx.x % p.n_xcd) * p.per_xcd + (int)(blockIdx.x / p.n_xcd);
    if (item < p.items) product_tile<KIND, false, false, EPI, ACT>(p, item, lds);
}

// The gate's gradient; the workgroups after the product's prepare the next
// launch, in the time that the last tiles leave compute units idle.
template <int KIND, int ACT>
__global__ __launch_bounds__(THREADS, per_cu(KIND)) void ff_gate_grad(FfProduct p, int32_t product_blocks, FfPrepare pre) {
    __shared__ __attribute__((aligned(256))) char lds[lds_bytes(KIND)];
    static_assert(COLUMN_LDS * 4 <= lds_bytes(KIND), "prepare_block's");
    if ((int)blockIdx.x >= product_blocks) {
        prepare_block(pre, (int)blockIdx.x - product_blocks, (float*)lds);
        return;
    }
    const int item = (int)(blockIdx.x % p.n_xcd) * p.per_xcd + (int)(blockIdx.x / p.n_xcd);
    if (item < p.items) product_tile<KIND, false, true, FF_GATE_GRAD, ACT>(p, item, lds);
}

// Up to three products of FF_STORE with W across the contraction in one
// launch (X across it too: the weights' gradients; or along it): their items
// together leave fewer compute units idle at the end than three launches do.
// The sums of the biases' gradients ride along.
struct FfGroup {
    FfProduct p[3];
    int32_t n;
    int32_t product_blocks;  // workgroups of the products; those after them do the sums
    PartialSums sums;
};
template <int KIND>
__global__ __launch_bounds__(THREADS, per_cu(KIND)) void ff_products(FfGroup g) {
    __shared__ __attribute__((aligned(256))) char lds[lds_bytes(KIND)];
    if ((int)blockIdx.x >= g.product_blocks) {
        sum_partials(g.sums, blockIdx.x - g.product_blocks, (float*)lds);
        return;
    }
    const int n_xcd = g.p[0].n_xcd;
    int j = blockIdx.x / n_xcd, which = 0;
    while (which < g.n - 1 && j >= g.p[which].per_xcd) j -= g.p[which++].per_xcd;
    const FfProduct& p = g.p[which];
    const int item = (int)(blockIdx.x % n_xcd) * p.per_xcd + j;
    if (item >= p.items) return;
    if (p.x_t)
        product_tile<KIND, true, true, FF_STORE, 0>(p, item, lds);
    else
        product_tile<KIND, false, true, FF_STORE, 0>(p, item, lds);
}

// out = the pieces' sums, in their order, + bias: eight outputs a thread.
struct FfSums {
    const float* part[3];
    const bf16* bias[3];
    bf16* out[3];
    int64_t n[3];          // outputs of a product, 0: none
    int32_t N[3], pieces[3];
};
__global__ __launch_bounds__(256) void ff_sum_pieces(FfSums a) {
    const int s = blockIdx.y;
    const int64_t i = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 8;
    if (i >= a.n[s]) return;
    float v[8], t[8];
    load8(a.part[s] + i, v);
    for (int k = 1; k < a.pieces[s]; ++k) {
        load8(a.part[s] + k * a.n[s] + i, t);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] += t[e];
    }
    if (a.bias[s] != nullptr) {
        load8(a.bias[s] + i % a.N[s], t);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] += t[e];
    }
    store8(a.out[s] + i, v);
}

int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

int64_t tiles_of(const FfProduct& p, int kind) {
    return ceil_div(p.M, rows_x(kind)) * ceil_div(p.N, outputs_of(kind, p.epilogue));
}

// Most pieces of a contraction, and most floats of all pieces' sums of a launch.
constexpr int kMaxPieces = 32;
constexpr int64_t kMaxPartFloats = 16 << 20;

// Pieces of a contraction in runs of about `run` k-tiles.
int64_t pieces_of(const FfProduct& p, int64_t run) {
    const int64_t n = (ceil_div(p.K, KT) + run / 2) / run;
    return n > 1 ? n : 1;
}

// Estimated us of n products on a kind of tile, their contractions in runs of
// about `run` k-tiles; floats: the pieces' sums.  By epilogue and kind: what a
// k-tile and an item (its start and epilogue) add to the longest item
// (kAlone) and to the busiest compute unit (kFull).
//
// These are weights for choosing, no times of a k-tile: FF_STORE's, kSlower (more
// k-tiles, lower clocks) and the pieces' cost were fitted until their choices
// came out fastest over the kinds and cuts measured for 39 sizes (77 to 16385
// tokens, 320 x 1280 to 2048 x 8192), 2 % above the best ones in the mean, 12 %
// at most.  (So the 256 x 256 tile's k-tile is 0.826 here, less than its 2048
// cycles of products.)  FF_GATE's and FF_GATE_GRAD's are round numbers set by
// hand; the latter's are TILE_64's, also where it runs as TILE_64_THREE.
struct TileCost {
    double tile, item;
};
constexpr TileCost kAlone[3][TILE_KINDS] = {{{0.307, 4.06}, {0.67, 4.24}, {1.55, 8.25}},
                                            {{0.31, 6.5}, {0.72, 12}},
                                            {{0.31, 10}, {0.72, 18}}};
constexpr TileCost kFull[3][TILE_KINDS] = {{{0.391, 1.74}, {0.548, 1.40}, {0.826, 10.8}},
                                           {{0.40, 2}, {0.95, 6}},
                                           {{0.40, 4.3}, {0.95, 18}}};
constexpr double kSlower[TILE_KINDS] = {0.067, 0.186, 0.412};
constexpr double kManyOutputs = 150.0 * 128 * 128;  // outputs x k-tiles of a compute unit
double estimate(const FfProduct* p, int n, int kind, int64_t run, int cus, int64_t& floats) {
    double work = 0, longest = 0, k_tiles = 0;
    int64_t items = 0;
    floats = 0;
    for (int i = 0; i < n; ++i) k_tiles += (double)ceil_div(p[i].K, KT) * tiles_of(p[i], kind);
    const double load = k_tiles * rows_x(kind) * rows_w(kind, p[0].epilogue) / cus / kManyOutputs;
    const double slower = p[0].epilogue == FF_STORE ? 1 + kSlower[kind] * (load < 1 ? load : 1) : 1;
    for (int i = 0; i < n; ++i) {
        const int64_t nkt = ceil_div(p[i].K, KT), pieces = pieces_of(p[i], run), t = tiles_of(p[i], kind) * pieces;
        const double len = (double)nkt / pieces;
        const TileCost &one = kAlone[p[i].epilogue][kind], &full = kFull[p[i].epilogue][kind];
        const double alone = len * one.tile + one.item;
        items += t;
        work += t * (len * full.tile * slower + full.item);
        if (alone > longest) longest = alone;
        if (pieces > 1) floats += pieces * p[i].M * p[i].N;
    }
    const double busiest = work / items * ceil_div(items, cus);  // of the compute units
    return (busiest > longest ? busiest : longest) + (floats > 0 ? 5.2 + 2.96e-6 * floats : 0);
}

int cus_here() {
    const int cus = device_cus();
    return cus > 0 ? cus : 256;
}

// The tile and the pieces of the products that are estimated fastest.
int plan(FfProduct* p, int n, int cus) {
    int64_t longest = 0;
    for (int i = 0; i < n; ++i) longest = longest > ceil_div(p[i].K, KT) ? longest : ceil_div(p[i].K, KT);
    int best_kind = TILE_128;
    int64_t best_run = longest;
    double best = 1e30;
    constexpr int kCuts[] = {1, 2, 3, 4, 6, 8, 12, 16, 24, kMaxPieces};
    for (int kind = 0; kind <= (p[0].epilogue == FF_STORE ? TILE_256 : TILE_128); ++kind)
        for (int cut : kCuts) {
            if (cut > 1 && p[0].epilogue != FF_STORE) break;
            const int64_t run = ceil_div(longest, cut);
            int64_t floats = 0;
            const double t = estimate(p, n, kind, run, cus, floats);
            if (floats > kMaxPartFloats || t >= best) continue;
            best = t;
            best_kind = kind;
            best_run = run;
        }
    const int n_xcd = layout_for(cus, cus).n_xcd;
    for (int i = 0; i < n; ++i) {
        p[i].pieces = (int32_t)pieces_of(p[i], best_run);
        p[i].items = (int32_t)(tiles_of(p[i], best_kind) * p[i].pieces);
        p[i].n_xcd = n_xcd;
        p[i].per_xcd = (p[i].items + n_xcd - 1) / n_xcd;
    }
    return best_kind;
}

// Places the sums of pieces in `part`.
void place_parts(FfProduct* p, int n, float* part) {
    for (int i = 0; i < n; ++i) {
        p[i].part = part;
        if (p[i].pieces > 1) part += (int64_t)p[i].pieces * p[i].M * p[i].N;
    }
}

hipError_t sum_pieces(const FfProduct* p, int n, hipStream_t s) {
    FfSums a = {};
    int k = 0;
    int64_t most = 0;
    for (int i = 0; i < n; ++i) {
        if (p[i].pieces == 1) continue;
        a.part[k] = p[i].part;
        a.bias[k] = p[i].bias;
        a.out[k] = p[i].out;
        a.n[k] = (int64_t)p[i].M * p[i].N;
        a.N[k] = p[i].N;
        a.pieces[k] = p[i].pieces;
        most = most > a.n[k] ? most : a.n[k];
        ++k;
    }
    if (k == 0) return hipSuccess;
    ff_sum_pieces<<<dim3((unsigned)ceil_div(most, 2048), k), 256, 0, s>>>(a);
    return hipGetLastError();
}

template <int KIND>
void launch(const FfProduct& p, hipStream_t s) {
    const unsigned grid = (unsigned)p.n_xcd * p.per_xcd;
    auto run = [&](auto kernel) { kernel<<<grid, THREADS, 0, s>>>(p); };
    if (p.epilogue == FF_STORE)
        run(ff_product<KIND, FF_STORE, 0>);
    else if constexpr (KIND != TILE_256)
        run(p.act == PCPP_ACT_SILU ? ff_product<KIND, FF_GATE, PCPP_ACT_SILU> : ff_product<KIND, FF_GATE, PCPP_ACT_GELU>);
}

bool skinny(const FfProduct& p) { return p.M <= FF_SKINNY_ROWS && !p.x_t && !p.w_t; }

}  // namespace

int ff_partial_rows(const FfProduct& p) {
    FfProduct q = p;
    return (int)(2 * ceil_div(p.M, rows_x(plan(&q, 1, cus_here()))));
}

int64_t ff_part_floats(const FfProduct* p, int n) {
    int64_t most = 0;
    for (int i = 0; i < n; ++i) {
        const int64_t nkt = ceil_div(p[i].K, KT);
        if (!skinny(p[i])) most += (nkt < kMaxPieces ? nkt : kMaxPieces) * p[i].M * p[i].N;
    }
    return most < kMaxPartFloats ? most : kMaxPartFloats;
}

void ff_plan(FfProduct* p, int n, int cus, int32_t* tile_rows, int32_t* tile_outputs) {
    if (cus <= 0) cus = cus_here();
    if (skinny(p[0])) {
        p[0].pieces = 1;
        *tile_rows = FF_SKINNY_ROWS;
        *tile_outputs = ff_skinny_outputs(p[0], cus);
        return;
    }
    const int kind = plan(p, n, cus);
    *tile_rows = rows_x(kind);
    *tile_outputs = outputs_of(kind, p[0].epilogue);
}

hipError_t launch_ff_product(FfProduct p, float* part, hipStream_t s) {
    if (skinny(p)) return launch_ff_skinny(p, cus_here(), s);
    const int kind = plan(&p, 1, cus_here());
    place_parts(&p, 1, part);
    if (kind == TILE_256)
        launch<TILE_256>(p, s);
    else if (kind == TILE_128)
        launch<TILE_128>(p, s);
    else
        launch<TILE_64>(p, s);
    const hipError_t e = hipGetLastError();
    return e != hipSuccess ? e : sum_pieces(&p, 1, s);
}

hipError_t launch_ff_gate_grad(FfProduct p, const FfPrepare& pre, hipStream_t s) {
    const int cus = cus_here(), kind = plan(&p, 1, cus);
    const unsigned blocks = (unsigned)p.n_xcd * p.per_xcd, grid = blocks + (unsigned)prepare_blocks(pre);
    auto run = [&](auto kernel) { kernel<<<grid, THREADS, 0, s>>>(p, (int32_t)blocks, pre); };
    const bool silu = p.act == PCPP_ACT_SILU;
    if (kind == TILE_128)
        run(silu ? ff_gate_grad<TILE_128, PCPP_ACT_SILU> : ff_gate_grad<TILE_128, PCPP_ACT_GELU>);
    else if (p.items > per_cu(TILE_64) * cus)
        run(silu ? ff_gate_grad<TILE_64_THREE, PCPP_ACT_SILU> : ff_gate_grad<TILE_64_THREE, PCPP_ACT_GELU>);
    else
        run(silu ? ff_gate_grad<TILE_64, PCPP_ACT_SILU> : ff_gate_grad<TILE_64, PCPP_ACT_GELU>);
    return hipGetLastError();
}

hipError_t launch_ff_products(const FfProduct* p, int n, float* part, const PartialSums& sums, hipStream_t s) {
    if (n == 0) return launch_sum_partials(sums, s);
    FfGroup g = {};
    g.sums = sums;
    g.n = n;
    for (int i = 0; i < n; ++i) {  // the longest contractions first
        int at = i;
        for (; at > 0 && g.p[at - 1].K < p[i].K; --at) g.p[at] = g.p[at - 1];
        g.p[at] = p[i];
    }
    const int kind = plan(g.p, n, cus_here());
    place_parts(g.p, n, part);
    unsigned grid = 0;
    for (int i = 0; i < n; ++i) grid += (unsigned)g.p[i].n_xcd * g.p[i].per_xcd;
    g.product_blocks = (int32_t)grid;
    grid += (unsigned)partial_sum_blocks(sums);
    if (kind == TILE_256)
        ff_products<TILE_256><<<grid, THREADS, 0, s>>>(g);
    else if (kind == TILE_128)
        ff_products<TILE_128><<<grid, THREADS, 0, s>>>(g);
    else
        ff_products<TILE_64><<<grid, THREADS, 0, s>>>(g);
    const hipError_t e = hipGetLastError();
    return e != hipSuccess ? e : sum_pieces(g.p, n, s);
}

}  // namespace pcpp

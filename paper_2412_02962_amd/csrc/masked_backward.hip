// Masked attention, backward: the gradient of the queries (masked_dq, a block
// of queries against all keys) and of keys and values (masked_dkv, a block of
// keys against the queries of all heads that read them), each computing the
// scores again.  Two kernels that own what they write, and so no atomics, for
// two more products than one that adds to dq from everywhere.  See
// masked_attention.h for the operands' layout.
//
// delta_i = dy_i . y_i takes y as it was rounded; the sum over the keys of P (dP -
// delta) is what it is off by, since that sum is 0.  masked_dq adds it up and
// leaves the better delta to masked_dkv, which runs after it.
//
// Five products of the forward's two, and the exponentials twice: bound by the
// vector unit and by waits for LDS, with 16 DB sums of 32 x 32 a lane (twice that
// for masked_dkv) leaving room for two wavefronts a SIMD and few operands ahead.
// 8192 causal, 16 heads of 128 on 4 of the keys: masked_dq 402 us (1025 TFLOP/s),
// masked_dkv 576 (955); capped and biased 538 and 697, the matrix unit busy for
// 31 % of the cycles in both, the vector unit for 56 and 44.  2 x 4096, 10 heads
// of 64: 159 (810) and 251 (685).
//
// P and dz are rounded to bf16, the matrix instructions' operands: half a step
// each, independent; the gradients are 0.0019 to 0.0024 off so, their own rounding
// 0.0017.  (Two bf16 each would double the products over keys and queries.)

#include <type_traits>

#include "masked_attention.h"

namespace pcpp {

using namespace masked;

namespace {

constexpr int NW = 4;
constexpr int NT = 64 * NW;
constexpr int BLOCK = 32 * NW;  // queries, or keys, of a workgroup

// delta = dy . y of a row: sixteen lanes to a row of a head.
__global__ __launch_bounds__(NT) void masked_delta(Params p) {
    const int lane = threadIdx.x & 15;
    const int64_t id = (int64_t)blockIdx.x * (NT / 16) + (threadIdx.x >> 4);
    if (id >= (int64_t)p.B * p.nq * p.H) return;
    const int64_t bi = id / p.H;
    const int head = (int)(id - bi * p.H), b = (int)(bi / p.nq), i = (int)(bi - (int64_t)b * p.nq);
    const int64_t at = b * p.y_batch + (int64_t)i * p.y_row + head * p.D + 8 * lane;
    float d = 0.f;
    if (8 * lane < p.D) {
        const bf16x8 a = *(const bf16x8*)(p.y + at), g = *(const bf16x8*)(p.dy + at);
#pragma unroll
        for (int e = 0; e < 8; ++e) d = __builtin_fmaf(bf16_to_f32(a[e]), bf16_to_f32(g[e]), d);
    }
#pragma unroll
    for (int s = 8; s > 0; s >>= 1) d += __shfl_xor(d, s);
    if (lane == 0) p.delta[((int64_t)b * p.H + head) * p.nq + i] = d;
}

template <int DB>
__device__ __forceinline__ void clear(f32x16 (&acc)[DB]) {
#pragma unroll
    for (int mb = 0; mb < DB; ++mb)
#pragma unroll
        for (int r = 0; r < 16; ++r) acc[mb][r] = 0.f;
}

template <int DB>
__device__ __forceinline__ void store_rows(bf16* row, const f32x16 (&acc)[DB], float f, int D, int lane) {
#pragma unroll
    for (int mb = 0; mb < DB; ++mb)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            if (32 * mb + 8 * g >= D) break;
            bf16x4 v;
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = f32_to_bf16(acc[mb][4 * g + e] * f);
            *(bf16x4*)(row + 32 * mb + 8 * g + 4 * (lane >> 5)) = v;
        }
}

// A row of gradients, or a piece's float32 part of it, in one pass over the
// registers.
template <int DB>
__device__ __forceinline__ void store_sums(bf16* row, float* part, const f32x16 (&acc)[DB], float f, int D, int lane) {
#pragma unroll
    for (int mb = 0; mb < DB; ++mb)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            const int c = 32 * mb + 8 * g;
            f32x4 v;
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = acc[mb][4 * g + e] * f;
            if (part != nullptr) {
                *(f32x4*)(part + c + 4 * (lane >> 5)) = v;
            } else if (c < D) {
                bf16x4 o;
#pragma unroll
                for (int e = 0; e < 4; ++e) o[e] = f32_to_bf16(v[e]);
                *(bf16x4*)(row + c + 4 * (lane >> 5)) = o;
            }
            __builtin_amdgcn_sched_barrier(0);  // (all products at once would be registers for all)
        }
}

constexpr float NEAR = 8.f;  // (in log2 units: a bias of a factor of 256)

template <int DB, bool CAP, bool BIAS>
__global__ __launch_bounds__(NT, DB <= 2 ? 3 : 2) void masked_dq(Params p) {
    using T = Tile<DB>;
    constexpr int SLOT = 2 * T::BYTES;  // K, V
    __shared__ __attribute__((aligned(16))) char lds[2 * SLOT];
    __shared__ __attribute__((aligned(16))) int docs[2][TILE];
    __shared__ Spoilt spoilt[NT];
    __shared__ uint32_t odd[2][NT];
    __shared__ DocRange kept[NW][64];
    const int tid = threadIdx.x, lane = tid & 63, half = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int nqb = (p.nq + BLOCK - 1) / BLOCK;
    const Place place = place_in(p.B * p.H, nqb, p.causal, p.kv_doc != nullptr);
    if (place.item < 0) return;
    const int bh = place.item, qb = nqb - 1 - place.block;
    const int b = scalar(bh / p.H), head = bh - b * p.H, kh = scalar(head / p.G);
    const Seq sq = seq_of(p, b);
    const int i0 = qb * BLOCK, last = min(i0 + BLOCK, p.nq) - 1;
    const int w0 = i0 + 32 * wave, wlast = min(w0 + 32, p.nq) - 1;
    const int i = w0 + (lane & 31), ic = min(i, p.nq - 1);
    const bool in = i < p.nq;
    const int pos = sq.pos0 + i, limit = limit_of(p, sq, i);
    const int doc = in && p.q_doc ? own_document(p.q_doc[(int64_t)b * p.nq + i]) : NO_DOC;
    const float slope2 = p.slopes ? p.slopes[head] * LOG2E : 0.f;
    const float lse2 = p.lse[(int64_t)bh * p.nq + ic] * LOG2E, delta = p.delta[(int64_t)bh * p.nq + ic];
    bf16x8 q[2 * DB], dy[2 * DB];
    load_rows<DB>(p.q + b * p.q_batch + (int64_t)ic * p.q_row + head * p.D, in, p.D, q, lane);
    load_rows<DB>(p.dy + b * p.y_batch + (int64_t)ic * p.y_row + head * p.D, in, p.D, dy, lane);

    const int end = tiles_of(limit_of(p, sq, last));
    const int lim_lo = limit_of(p, sq, w0), lim_hi = w0 <= wlast ? limit_of(p, sq, wlast) : 0;
    const int least = limit_of(p, sq, i0);  // every query sees the keys before (documents apart)
    DocWindow window;
    {
        DocRange all = {}, mine = {};
        if (p.kv_doc) {
            mine = range_of_lanes(doc, in);
            const DocRange* r = p.q_range + (int64_t)b * tiles_of(p.nq) + i0 / TILE;
            all = r[0];
            if (last / TILE > i0 / TILE) all = joined(all, r[1]);
        }
        window.init(p.kv_range + (int64_t)b * tiles_of(p.nkv), kept[wave], end, all, mine, p.kv_doc != nullptr);
    }
    const Loader<DB, NW, TILE> kload(p.k_row, p.D, wave, lane), vload(p.v_row, p.D, wave, lane);
    const Reader<DB> reader(lane);
    const bf16* kb = p.k + b * p.k_batch + kh * p.D;
    const bf16* vb = p.v + b * p.v_batch + kh * p.D;
    const uint32_t lds0 = lds_address(lds);
    int dr = -1;
    auto issue = [&](int t, int slot) {
        kload.issue(kb, t * TILE, sq.len, lds0 + slot * SLOT);
        vload.issue(vb, t * TILE, sq.len, lds0 + slot * SLOT + T::BYTES);
        if (p.kv_doc && tid < TILE) dr = t * TILE + tid < sq.len ? max(p.kv_doc[(int64_t)b * p.nkv + t * TILE + tid], -1) : -1;
    };
    if (2 * p.D < T::RB) {
        clear_tiles(lds, 2 * SLOT, NT);
        __syncthreads();
    }

    f32x16 acc[DB];
    float off = 0.f;  // sum of P (dP - delta)
    auto step = [&](const char* kt, const int* dt, int row0, int j0, bool partial, bool cleaned) __attribute__((always_inline)) {
        const char* vt = kt + T::BYTES;
        const Reader<DB> rd = reader.template fresh<CAP>();
        f32x16 s, dp;
        staged<4 * DB, 2>([&](int i) __attribute__((always_inline)) { return rd.rows(i & 1 ? vt : kt, row0, i >> 1); },
                           [&](int i, const bf16x8& x) __attribute__((always_inline)) {
                               const int kk = i >> 1;
                               if (i & 1)
                                   dp = mfma32x32x16(x, dy[kk], kk == 0 ? f32x16{} : dp);
                               else
                                   s = mfma32x32x16(x, q[kk], kk == 0 ? f32x16{} : s);
                           });
        if (cleaned) put_scores(odd[row0 / 32][threadIdx.x], s);
        const int base = j0 + 4 * half;
        const float far = (float)(pos - base);
        float w[16];
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            float slope, x = score<CAP>(p, s[r], -lse2, &slope);
            if constexpr (BIAS) x = __builtin_fmaf(-slope2, fabsf(far - (float)(8 * (r >> 2) + (r & 3))), x);
            w[r] = fast_exp2(x) * (dp[r] - delta);
            if constexpr (CAP) dp[r] = slope;
        }
        if (partial) {
            // (the derivative too: it is NaN where the key is)
            auto keep = [&](int r, bool seen) __attribute__((always_inline)) {
                w[r] = seen ? w[r] : 0.f;
                if constexpr (CAP) dp[r] = seen ? dp[r] : 0.f;
            };
            int lim = limit - base;
            asm volatile("" : "+v"(lim));  // (a branch, not selections in every step)
#pragma unroll
            for (int r = 0; r < 16; ++r) keep(r, 8 * (r >> 2) + (r & 3) < lim);
            if (p.kv_doc) {
                int at = row0 + 4 * half;
                asm volatile("" : "+v"(at));
#pragma unroll
                for (int g = 0; g < 4; ++g) {
                    const i32x4 d = *(const i32x4*)(dt + at + 8 * g);
#pragma unroll
                    for (int e = 0; e < 4; ++e) keep(4 * g + e, d[e] == doc);
                }
            }
        }
        bf16x8 o[1][2];
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            off += w[r];
            if constexpr (CAP) w[r] *= dp[r];
            o[0][r >> 3][r & 7] = f32_to_bf16(w[r]);
        }
        add_rows<DB, 1>(acc, o, rd, kt, row0);
        if constexpr (BIAS) {
            // A bias rests a query on the few keys near it, and there y's own
            // rounding (in delta) is seen in dq.  The weights' is taken out for
            // them, so that the two do not add up.
            const int apart = max(j0 - pos, pos - j0 - 31);
            const bool near = slope2 > 0.f && slope2 * (float)apart < NEAR;
            if (__any(near)) {
#pragma unroll
                for (int r = 0; r < 16; ++r) w[r] = near ? w[r] - bf16_to_f32(o[0][r >> 3][r & 7]) : 0.f;
                pack(w, o[0]);
                add_rows<DB, 1>(acc, o, rd, kt, row0);
            }
        }
    };

    spoilt[tid] = Spoilt{0, 0};
    clear<DB>(acc);
    int slot = 0, t = window.next(0);
    bool same = true, apart = false, same_all = true;
    auto look = [&](int of, bool& a, bool& b_, bool& c_) { a = window.same(of), b_ = window.apart(of), c_ = window.same_all(of); };
    if (t < end) {
        look(t, same, apart, same_all);
        issue(t, slot);
    }
    while (t < end) {
        landed();
        if (p.kv_doc && tid < TILE) docs[slot][tid] = dr;
        __syncthreads();  // the tile is there, and nobody reads the one before any more
        const int tn = window.next(t + 1);
        bool same_n = true, apart_n = false, same_all_n = true;
        if (tn < end) {
            look(tn, same_n, apart_n, same_all_n);
            issue(tn, slot ^ 1);
        }
        char* kt = lds + slot * SLOT;
        bool cleaned = false;
        if ((t + 1) * TILE > least || !same_all) {
            bool bad = false;
#pragma unroll
            for (int o = 0; o < T::BYTES; o += 16 * NT) bad |= not_finite16(kt + o + 16 * tid);
            cleaned = scalar(__syncthreads_or(bad));
            if (cleaned) {
                int row = w0 + (lane & 31);
                asm volatile("" : "+v"(row));  // (worked out here)
                const bf16* own = p.q + b * p.q_batch + (int64_t)min(row, p.nq - 1) * p.q_row + head * p.D;
#pragma unroll 1
                for (int h = 0; h < 2; ++h) {
                    uint32_t seen = 0;
#pragma unroll 1
                    for (int j = 0; j < 32; ++j)
                        seen |= (uint32_t)((t * TILE + 32 * h + j < limit) & (!p.kv_doc || docs[slot][32 * h + j] == doc)) << j;
                    const uint32_t rows = spoilt_rows<DB>(kt, 32 * h, seen, lane);
                    note_spoilt<DB>(spoilt + tid, kt, 32 * h, rows, seen, lane);
                    odd[h][tid] = note_scores<DB>(kt, 32 * h, rows, own, p.D, lane);
                }
                __syncthreads();
                for (int o = 0; o < T::BYTES; o += 16 * NT) make_finite16(kt + o + 16 * tid);
                __syncthreads();
            }
        }
#pragma unroll 1
        for (int h = 0; h < 2; ++h) {
            const int j0 = t * TILE + 32 * h;
            if (j0 >= lim_hi || apart) continue;
            step(kt, docs[slot], 32 * h, j0, j0 + 32 > lim_lo || !same, cleaned);
        }
        t = tn, same = same_n, apart = apart_n, same_all = same_all_n;
        slot ^= 1;
    }
    // (a key with an infinity: its score is infinite, and dz 0, by the cap or by P, or NaN)
    put_spoilt<DB>(spoilt + tid, acc, true);
    off = sum_halves(off);
    if (!in) return;
    if (lane < 32) {
        p.delta[(int64_t)bh * p.nq + i] = -(delta + off);
        p.lse2[(int64_t)bh * p.nq + i] = -lse2;
    }
    if (p.dq) store_rows<DB>(p.dq + b * p.q_batch + (int64_t)i * p.q_row + head * p.D, acc, CAP ? 4.f * p.scale : p.scale, p.D, lane);
}

// What a tile's queries bring besides q and dy, as masked_dq left it.
template <int ROWS>
struct QueryTile {
    float lse2[ROWS], delta[ROWS];
    int doc[ROWS];
};

// A block of keys against a piece of the queries (of all heads that read them,
// one head after the other).  Up to 64 channels: K and V in registers, tiles of
// 64 queries; above, where the two sums alone take half the registers that two
// wavefronts of a SIMD have, V in LDS and tiles of 32 queries.
template <int DB, bool CAP, bool BIAS>
__global__ __launch_bounds__(NT, 2) void masked_dkv(Params p) {
    using T = Tile<DB>;
    constexpr int ROWS = DB <= 2 ? 64 : 32, TB = ROWS * T::RB;
    constexpr int SLOT = 2 * TB;  // Q, dy
    constexpr bool V_LDS = DB > 2;
    constexpr int LDS = 2 * SLOT + (V_LDS ? BLOCK * T::RB : 0);
    __shared__ __attribute__((aligned(16))) char lds[LDS];
    __shared__ __attribute__((aligned(16))) QueryTile<ROWS> brought[2];
    __shared__ Spoilt spoilt_v[NT], spoilt_k[NT];
    __shared__ uint32_t odd[ROWS / 32][NT];
    __shared__ DocRange kept[NW][64];
    const int tid = threadIdx.x, lane = tid & 63, half = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int nkb = (p.nkv + BLOCK - 1) / BLOCK;
    const Place place = place_in(p.B * p.KH * p.pieces, nkb, p.causal, false);
    if (place.item < 0) return;
    const int item = place.item, kb = place.block;  // (the first keys are seen by the most)
    const int bk = scalar(item / p.pieces), piece = item - bk * p.pieces;
    const int b = scalar(bk / p.KH), kh = bk - b * p.KH;
    const Seq sq = seq_of(p, b);
    const int k0 = kb * BLOCK, klast = min(k0 + BLOCK, p.nkv) - 1;
    const int w0 = k0 + 32 * wave;
    const int j = w0 + (lane & 31);
    const bool in = j < p.nkv, live = j < sq.len;
    const int doc = live && p.kv_doc ? own_document(p.kv_doc[(int64_t)b * p.nkv + j]) : NO_DOC;
    // The queries that see key j by length, past and prefix: from .. nq - 1.
    const int from = !live || (p.kv_doc && doc == NO_DOC) ? p.nq : !p.causal || j < sq.prefix ? 0 : min(max(j - sq.pos0, 0), p.nq);
    if (V_LDS || 2 * p.D < T::RB) {
        clear_tiles(lds, LDS, NT);
        __syncthreads();
    }
    bf16x8 k[2 * DB], v[V_LDS ? 1 : 2 * DB];
    load_rows<DB>(p.k + b * p.k_batch + (int64_t)min(j, p.nkv - 1) * p.k_row + kh * p.D, live, p.D, k, lane);
    const bf16* vrow = p.v + b * p.v_batch + (int64_t)min(j, p.nkv - 1) * p.v_row + kh * p.D;
    const Reader<DB> reader(lane);
    char* vt = lds + 2 * SLOT;  // all of the block's keys
    if constexpr (V_LDS) {
        bf16x8 x[2 * DB];
        load_rows<DB>(vrow, live, p.D, x, lane);
#pragma unroll
        for (int kk = 0; kk < 2 * DB; ++kk) *(bf16x8*)(vt + 32 * wave * T::RB + (reader.row_at ^ (32 * kk))) = x[kk];
    } else {
        load_rows<DB>(vrow, live, p.D, v, lane);
    }

    // Tiles of ROWS queries: this piece's, in order of heads and queries.
    const int nt = (p.nq + ROWS - 1) / ROWS;
    int first = 0;  // tile of the first query that sees the block's first key
    if (p.causal && k0 >= sq.prefix) first = min(max(k0 - sq.pos0, 0), p.nq) / ROWS;
    if (k0 >= sq.len) first = nt;
    const int tiles = nt - min(first, nt);
    const int64_t all_tiles = (int64_t)tiles * p.G;
    const int u0 = scalar((int)(all_tiles * piece / p.pieces)), u1 = scalar((int)(all_tiles * (piece + 1) / p.pieces));
    DocWindow window;
    {
        DocRange all = {}, mine = {};
        if (p.kv_doc) {
            mine = range_of_lanes(doc, live);
            const DocRange* r = p.kv_range + (int64_t)b * tiles_of(p.nkv) + k0 / TILE;
            all = r[0];
            if (klast / TILE > k0 / TILE) all = joined(all, r[1]);
        }
        window.init(p.q_range + (int64_t)b * tiles_of(p.nq), kept[wave], tiles_of(p.nq), all, mine, p.kv_doc != nullptr);
    }
    // The first tile from t on that may have the block's documents.
    auto next = [&](int t) {
        const int w = window.next(t * ROWS / TILE);
        return w == t * ROWS / TILE ? t : w * (TILE / ROWS);
    };

    const Loader<DB, NW, ROWS> qload(p.q_row, p.D, wave, lane), gload(p.y_row, p.D, wave, lane);
    const uint32_t lds0 = lds_address(lds);
    const uint32_t brought0 = lds_address(brought);
    auto issue = [&](int g, int t, int slot) {
        const int head = kh * p.G + g;
        qload.issue(p.q + b * p.q_batch + head * p.D, t * ROWS, p.nq, lds0 + slot * SLOT);
        gload.issue(p.dy + b * p.y_batch + head * p.D, t * ROWS, p.nq, lds0 + slot * SLOT + TB);
        if (tid < ROWS) {
            const uint32_t at = 4 * min(tid, p.nq - 1 - t * ROWS), to = brought0 + slot * sizeof(QueryTile<ROWS>);
            const int64_t row = ((int64_t)b * p.H + head) * p.nq + t * ROWS;
            load_lds4(uniform64((uint64_t)(uintptr_t)(p.lse2 + row)), at, to);
            load_lds4(uniform64((uint64_t)(uintptr_t)(p.delta + row)), at, to + 4 * ROWS);
            if (p.q_doc) load_lds4(uniform64((uint64_t)(uintptr_t)(p.q_doc + (int64_t)b * p.nq + t * ROWS)), at, to + 8 * ROWS);
        }
    };

    f32x16 dk[DB], dv[DB];
    auto step = [&](const char* qt, const QueryTile<ROWS>& rows, int row0, int i0, float slope2, bool partial,
                    bool cleaned) __attribute__((always_inline)) {
        const char* gt = qt + TB;
        const Reader<DB> rd = reader.fresh();
        f32x16 s, dp;
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            const f32x4 d = *(const f32x4*)(rows.delta + row0 + 8 * g + 4 * half);
#pragma unroll
            for (int e = 0; e < 4; ++e) dp[4 * g + e] = d[e];
        }
        // q for s, and dy with v for dp, in turn
        struct Operands {
            bf16x8 a, b;
        };
        staged<4 * DB, (DB > 3 ? 1 : 2)>(
            [&](int i) __attribute__((always_inline)) {
                Operands o;
                o.a = rd.rows(i & 1 ? gt : qt, row0, i >> 1);
                if constexpr (V_LDS)
                    if (i & 1) o.b = rd.rows(vt, 32 * wave, i >> 1);
                return o;
            },
            [&](int i, const Operands& o) __attribute__((always_inline)) {
                const int kk = i >> 1;
                if ((i & 1) == 0)
                    s = mfma32x32x16(o.a, k[kk], kk == 0 ? f32x16{} : s);
                else if constexpr (V_LDS)
                    dp = mfma32x32x16(o.a, o.b, dp);
                else
                    dp = mfma32x32x16(o.a, v[kk], dp);
            });
        if (cleaned) put_scores(odd[row0 / 32][threadIdx.x], s);
        const int base = i0 + 4 * half;
        const float far = (float)(sq.pos0 + base - j);
        float w[16], z[16];
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            const f32x4 lse2 = *(const f32x4*)(rows.lse2 + row0 + 8 * g + 4 * half);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int r = 4 * g + e;
                float slope, x = score<CAP>(p, s[r], lse2[e], &slope);
                if constexpr (BIAS) x = __builtin_fmaf(-slope2, fabsf(far + (float)(8 * g + e)), x);
                w[r] = fast_exp2(x);
                z[r] = w[r] * dp[r];
                if constexpr (CAP) z[r] *= slope;
            }
        }
        if (partial) {
            auto keep = [&](int r, bool seen) __attribute__((always_inline)) {
                w[r] = seen ? w[r] : 0.f;
                z[r] = seen ? z[r] : 0.f;
            };
            uint32_t lo = from - base;
            const uint32_t n = max(p.nq - from, 0);  // rows lo .. lo + n - 1, in one comparison
            asm volatile("" : "+v"(lo));             // (a branch, not selections in every step)
#pragma unroll
            for (int r = 0; r < 16; ++r) keep(r, (uint32_t)(8 * (r >> 2) + (r & 3)) - lo < n);
            if (p.kv_doc) {
                int at = row0 + 4 * half;
                asm volatile("" : "+v"(at));
#pragma unroll
                for (int g = 0; g < 4; ++g) {
                    const i32x4 d = *(const i32x4*)(rows.doc + at + 8 * g);
#pragma unroll
                    for (int e = 0; e < 4; ++e) keep(4 * g + e, d[e] == doc);
                }
            }
        }
        bf16x8 o[1][2];
        if constexpr (DB > 3) __builtin_amdgcn_sched_barrier(0);
        pack(w, o[0]);
        add_rows<DB, 1>(dv, o, rd, gt, row0);
        if constexpr (DB > 3) __builtin_amdgcn_sched_barrier(0);
        pack(z, o[0]);
        add_rows<DB, 1>(dk, o, rd, qt, row0);
    };

    spoilt_v[tid] = spoilt_k[tid] = Spoilt{0, 0};
    clear<DB>(dk);
    clear<DB>(dv);
    int slot = 0, g = 0, t = 0;
    bool more = u0 < u1, same = true, apart = false, same_all = true;
    // From tile t of head g on: the first that counts, and whether this piece has it.
    auto settle = [&](int& hg, int& ht) {
        while (hg < p.G) {
            ht = next(ht);
            if (ht < nt) return hg * tiles + ht - first < u1;
            ++hg;
            ht = first;
        }
        return false;
    };
    auto look = [&](int ht, bool& a, bool& c, bool& d) {
        const int w = ht * ROWS / TILE;
        a = window.same(w), c = window.apart(w), d = window.same_all(w);
    };
    if (more) {
        g = scalar(u0 / tiles);
        t = first + u0 - g * tiles;
        more = settle(g, t);
    }
    if (more) {
        look(t, same, apart, same_all);
        issue(g, t, slot);
    }
    while (more) {
        landed();
        __syncthreads();  // the tile is there, and nobody reads the one before any more
        int gn = g, tn = t + 1;
        const bool more_n = settle(gn, tn);
        bool same_n = true, apart_n = false, same_all_n = true;
        if (more_n) {
            look(tn, same_n, apart_n, same_all_n);
            issue(gn, tn, slot ^ 1);
        }
        const float slope2 = BIAS && p.slopes ? p.slopes[kh * p.G + g] * LOG2E : 0.f;
        char* qt = lds + slot * SLOT;
        const int i0 = t * ROWS;
        bool cleaned = false;
        if (i0 + ROWS > p.nq || k0 + BLOCK > limit_of(p, sq, i0) || !same_all) {
            bool bad = false;
#pragma unroll 1
            for (int o = 0; o < SLOT; o += 16 * NT) bad |= not_finite16(qt + o + 16 * tid);
            cleaned = scalar(__syncthreads_or(bad));
            if (cleaned) {
                int row = j;
                asm volatile("" : "+v"(row));  // (worked out here)
                const bf16* own = p.k + b * p.k_batch + (int64_t)min(row, sq.len - 1) * p.k_row + kh * p.D;
#pragma unroll 1
                for (int h = 0; h < ROWS; h += 32) {
                    uint32_t seen = 0;
                    for (int r = 0; r < 32; ++r) {
                        const int i = i0 + h + r, d = brought[slot].doc[h + r];
                        seen |= (uint32_t)((i >= from) & (i < p.nq) & (!p.kv_doc || d == doc)) << r;
                    }
                    note_spoilt<DB>(spoilt_v + tid, qt + TB, h, spoilt_rows<DB>(qt + TB, h, seen, lane), seen, lane);
                    const uint32_t rows = spoilt_rows<DB>(qt, h, seen, lane);
                    note_spoilt<DB>(spoilt_k + tid, qt, h, rows, seen, lane);
                    odd[h / 32][tid] = note_scores<DB>(qt, h, rows, own, p.D, lane);
                }
                // (dP needs no note: a query whose dy is not finite has NaN in its delta)
                __syncthreads();
                for (int o = 0; o < SLOT; o += 16 * NT) make_finite16(qt + o + 16 * tid);
                __syncthreads();
            }
        }
#pragma unroll 1
        for (int h = 0; h < ROWS; h += 32) {
            const int ih = i0 + h;
            if (apart || ih >= p.nq || w0 >= limit_of(p, sq, min(ih + 31, p.nq - 1))) continue;
            step(qt, brought[slot], h, ih, slope2, ih + 32 > p.nq || w0 + 32 > limit_of(p, sq, ih) || !same,
                 cleaned);
        }
        g = gn, t = tn, same = same_n, apart = apart_n, same_all = same_all_n, more = more_n;
        slot ^= 1;
    }
    put_spoilt<DB>(spoilt_v + tid, dv);
    // (a query with an infinity: its scores are infinite, and dz 0, by the cap, or NaN)
    put_spoilt<DB>(spoilt_k + tid, dk, true);
    if (!in) return;
    constexpr int CH = 32 * DB;
    float* part = p.pieces > 1 ? p.part_o + (((int64_t)piece * p.B * p.KH + bk) * p.nkv + j) * (2 * CH) : nullptr;
    store_sums<DB>(p.dk + b * p.k_batch + (int64_t)j * p.k_row + kh * p.D, part, dk, CAP ? 4.f * p.scale : p.scale, p.D, lane);
    store_sums<DB>(p.dv + b * p.v_batch + (int64_t)j * p.v_row + kh * p.D, part ? part + CH : nullptr, dv, 1.f, p.D, lane);
}

// The pieces' sums, in their order: eight channels of dk or dv of a key a thread.
__global__ __launch_bounds__(NT) void masked_join_kv(Params p, int CH) {
    const int per = 2 * CH / 8;
    const int64_t id = (int64_t)blockIdx.x * NT + threadIdx.x, rows = (int64_t)p.B * p.KH * p.nkv;
    const int64_t row = id / per;
    if (row >= rows) return;
    const int c = 8 * (int)(id - row * per);
    const float* in = p.part_o + row * (2 * CH) + c;
    f32x4 a = {}, b4 = {};
    for (int k = 0; k < p.pieces; ++k) {
        a += *(const f32x4*)(in + k * rows * (2 * CH));
        b4 += *(const f32x4*)(in + k * rows * (2 * CH) + 4);
    }
    const int64_t bk = row / p.nkv;
    const int j = (int)(row - bk * p.nkv), b = (int)(bk / p.KH), kh = (int)(bk - (int64_t)b * p.KH);
    const int ch = c < CH ? c : c - CH;
    if (ch >= p.D) return;
    bf16* o = c < CH ? p.dk + b * p.k_batch + (int64_t)j * p.k_row : p.dv + b * p.v_batch + (int64_t)j * p.v_row;
    bf16x8 v;
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = f32_to_bf16(a[e]), v[4 + e] = f32_to_bf16(b4[e]);
    *(bf16x8*)(o + kh * p.D + ch) = v;
}

}  // namespace

hipError_t launch_masked_delta(const Params& p, hipStream_t s) {
    const int64_t rows = (int64_t)p.B * p.nq * p.H;
    masked_delta<<<(unsigned)((rows + NT / 16 - 1) / (NT / 16)), NT, 0, s>>>(p);
    return hipGetLastError();
}

hipError_t launch_masked_dq(const Params& p, hipStream_t s) {
    const int64_t blocks = (int64_t)p.B * p.H * ((p.nq + BLOCK - 1) / BLOCK);
    return with_shape(p, [&](auto db, auto cap, auto bias) {
        masked_dq<db(), cap(), bias()><<<blocks_for(blocks), NT, 0, s>>>(p);
        return hipGetLastError();
    });
}

hipError_t launch_masked_dkv(const Params& p, hipStream_t s) {
    const int64_t blocks = (int64_t)p.B * p.KH * ((p.nkv + BLOCK - 1) / BLOCK) * p.pieces;
    const hipError_t e = with_shape(p, [&](auto db, auto cap, auto bias) {
        masked_dkv<db(), cap(), bias()><<<blocks_for(blocks), NT, 0, s>>>(p);
        return hipGetLastError();
    });
    if (e != hipSuccess || p.pieces == 1) return e;
    const int ch = 32 * blocks_of(p.D);
    const int64_t threads = (int64_t)p.B * p.KH * p.nkv * (2 * ch / 8);
    masked_join_kv<<<(unsigned)((threads + NT - 1) / NT), NT, 0, s>>>(p, ch);
    return hipGetLastError();
}

}  // namespace pcpp

// Masked attention, forward: many queries (masked_forward), and few queries on
// many keys (masked_few, masked_join).  See masked_attention.h for the
// operands' layout.
//
// Scores are computed transposed, S^T = K Q^T, a query to a lane: its maximum,
// its sum and its mask are a lane's own, and P^T is the operand of y^T = V^T P^T
// as it stands.  The maximum is taken only when a lane's probabilities of a
// step's keys sum to 2^20 or more (or to no number): until then the one before
// serves, which saves its exchange between the halves of the wavefront and the
// results' factor in nearly every step.  A step is 64 keys, so that the products
// of some run under the exponentials of others (8192 queries and keys, bf16: 16
// heads of 64 337 us, 32 keys a step 402; of 128 562, else 654).
//
// The probabilities are rounded to bf16, the matrix instructions' operands: up to
// half a step each, independent.  y is 0.0019 to 0.0024 off so, its own rounding
// 0.0017.  (Two bf16 each, as masked_few has them, are twice the products.)
//
// Bound by the vector unit and the wavefronts' own waits, two or three of them to
// a SIMD: 8192 causal, 16 heads of 128 on 4 of the keys, capped and biased
// (three transcendental operations a score), with lse 389 us and 705 TFLOP/s, the
// matrix unit busy for 28 % of the cycles and the vector unit for 58; without cap
// and bias 301 us, 915 TFLOP/s, without lse too 289, 950; not causal, 16 heads of
// keys too, 550 us, 1000 (with lse 572).

#include <type_traits>

#include "masked_attention.h"

namespace pcpp {

using namespace masked;

namespace {

constexpr float P_LIMIT = 1048576.0f;
constexpr int NW = 4;
constexpr int NT = 64 * NW;
constexpr int QB = 32 * NW;  // queries of a workgroup of masked_forward

// A lane's query.
struct Row {
    int pos, limit;       // limit: it sees no key from here on
    int doc;              // NO_DOC: none
    float slope2;         // of the bias, log2 units
};

// Running maximum (log2 units), sum and result of the lanes' queries; `exact`:
// the sum of the probabilities as they were before their rounding to bf16.
template <int DB>
struct State {
    float m, l, exact;
    f32x16 o[DB];
};
template <int DB>
__device__ __forceinline__ void clear(State<DB>& st) {
    st.m = -INFINITY;
    st.l = st.exact = 0.f;
#pragma unroll
    for (int mb = 0; mb < DB; ++mb)
#pragma unroll
        for (int r = 0; r < 16; ++r) st.o[mb][r] = 0.f;
}

// What is the same in every step of a wavefront.
template <int DB>
struct Context {
    const Params& p;
    const bf16x8 (&q)[2 * DB];
    const Row& row;
    const Reader<DB>& rd;
    int lane;
};

// 32 HB keys from key j0, the tiles' first rows.  partial: some query does
// not see some key.  TWO: the probabilities as two bf16 (for few queries, where
// the products cost nothing and a token's error counts).
// EXACT: the sum for lse too.  y is divided by the sum of the rounded
// probabilities: where one key dominates, the rounding of its weight is above
// and below the line and cancels.  In lse nothing would cancel it: off by up to
// 2^-8 there, and with it all of the row's probabilities in the backward pass.
// (Without lse and with it, us: 8192 causal, 16 heads of 128 on 4, 289 and 301;
// 8192, 16 heads of 64, 343 and 364; packed documents 67.2 and 67.0.)
// after_scores: what may run once the keys have been used.
template <int DB, int HB, bool CAP, bool BIAS, bool TWO, bool EXACT, typename After>
__device__ __forceinline__ void step(const Context<DB>& c, State<DB>& st, const char* kt, const char* vt, const int* docs, int j0,
                                     bool partial, bool first, After after_scores) {
    const Params& p = c.p;
    const Row& row = c.row;
    const Reader<DB> rd = c.rd.fresh();
    const int half = c.lane >> 5;
    const int base = j0 + 4 * half;
    const float far = (float)(row.pos - base);
    // Mostly once round.  Where the probabilities by the maximum so far are too
    // large, a second time for the scores' maximum and a third by that one (the
    // scores are computed again: registers for them would be held all along).
    // The first step of all begins with the maximum.
    bool search = first, tried = false;
    float w[HB][16];
    bf16x8 pr[HB][2];
    float sum, exact;
    uint32_t over = search ? ~0u : 0u;  // the lanes that need another maximum
#pragma unroll 1
    for (;;) {
        f32x16 s[HB];
        staged<2 * DB * HB, 2>([&](int i) __attribute__((always_inline)) { return rd.rows(kt, 32 * (i / (2 * DB)), i % (2 * DB)); },
                               [&](int i, const bf16x8& k) __attribute__((always_inline)) {
                                   const int h = i / (2 * DB), kk = i % (2 * DB);
                                   s[h] = mfma32x32x16(k, c.q[kk], kk == 0 ? f32x16{} : s[h]);
                               });
        // Scores less the maximum, in log2 units; -infinity where not seen (also
        // while the maximum is still -infinity and all others are infinite).
        const float add = search ? 0.f : -st.m;
#pragma unroll
        for (int h = 0; h < HB; ++h)
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                w[h][r] = score<CAP>(p, s[h][r], add);
                if constexpr (BIAS) w[h][r] = __builtin_fmaf(-row.slope2, fabsf(far - (float)(32 * h + 8 * (r >> 2) + (r & 3))), w[h][r]);
            }
        if (partial) {
            int limit = row.limit - base;
            asm volatile("" : "+v"(limit));  // (a branch, not selections in every step)
#pragma unroll
            for (int h = 0; h < HB; ++h)
#pragma unroll
                for (int r = 0; r < 16; ++r) w[h][r] = 32 * h + 8 * (r >> 2) + (r & 3) < limit ? w[h][r] : -INFINITY;
            if (p.kv_doc) {
                int at = 4 * half;
                asm volatile("" : "+v"(at));
#pragma unroll
                for (int g = 0; g < 4 * HB; ++g) {
                    const i32x4 d = *(const i32x4*)(docs + at + 8 * g);
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        float& x = w[g >> 2][4 * (g & 3) + e];
                        x = max(d[e], -1) == row.doc ? x : -INFINITY;
                    }
                }
            }
        }
        if (search) {
            float mx = w[0][0];
#pragma unroll
            for (int h = 0; h < HB; ++h)
#pragma unroll
                for (int r = 0; r < 16; ++r) mx = fmaxf(mx, w[h][r]);
            // (each query by its own sums: what others see is nothing to it)
            const float m_new = over ? fmaxf(st.m, max_halves(mx)) : st.m;
            const float alpha = m_new == st.m ? 1.f : fast_exp2(st.m - m_new);
            st.m = m_new;
            st.l *= alpha;
            if constexpr (EXACT) st.exact *= alpha;
#pragma unroll
            for (int mb = 0; mb < DB; ++mb)
#pragma unroll
                for (int r = 0; r < 16; ++r) st.o[mb][r] *= alpha;
            search = false;
            over = 0;
            tried = true;
            continue;
        }
        sum = exact = 0.f;
#pragma unroll
        for (int h = 0; h < HB; ++h)
#pragma unroll
            for (int r = 0; r < 16; r += 2) {
                float &a = w[h][r], &b = w[h][r + 1];
                a = fast_exp2(a);
                b = fast_exp2(b);
                const bf16x2 pk = {f32_to_bf16(a), f32_to_bf16(b)};
                pr[h][r >> 3][r & 7] = pk[0];
                pr[h][r >> 3][(r & 7) + 1] = pk[1];
                if constexpr (TWO)
                    sum += a + b;
                else
                    sum = __builtin_amdgcn_fdot2_f32_bf16(pk, bf16x2{(bf16)1.f, (bf16)1.f}, sum, false);
                if constexpr (EXACT) exact += a + b;
            }
        if constexpr (EXACT) asm volatile("" : "+v"(exact));  // (here, not behind the loop with all of w for it)
        if (tried || !__any(!(sum < P_LIMIT))) break;
        over = max_halves(sum < P_LIMIT ? 0.f : 1.f) > 0.f;
        search = true;
    }
    after_scores();
    st.l += sum;
    if constexpr (EXACT) st.exact += exact;
    add_rows<DB, HB>(st.o, pr, rd, vt, 0);
    if constexpr (TWO) {
        static_assert(HB == 1, "few queries");
#pragma unroll
        for (int r = 0; r < 16; ++r) w[0][r] -= bf16_to_f32(pr[0][r >> 3][r & 7]);
        pack(w[0], pr[0]);
        add_rows<DB, HB>(st.o, pr, rd, vt, 0);
    }
}

// Which of the 32 keys from j0 the lane's query sees.
__device__ __forceinline__ uint32_t keys_seen(const Params& p, const Row& row, const int* docs, int j0) {
    uint32_t seen = 0;
#pragma unroll 1
    for (int j = 0; j < 32; ++j)
        seen |= (uint32_t)((j0 + j < row.limit) & (!p.kv_doc || max(docs[j], -1) == row.doc)) << j;
    return seen;
}

__device__ __forceinline__ Row row_of(const Params& p, const Seq& sq, int b, int head, int i, bool in) {
    Row r;
    r.pos = sq.pos0 + i;
    r.limit = limit_of(p, sq, i);
    r.doc = in && p.q_doc ? own_document(p.q_doc[(int64_t)b * p.nq + i]) : NO_DOC;
    r.slope2 = p.slopes ? p.slopes[head] * LOG2E : 0.f;
    return r;
}

template <int DB, bool CAP, bool BIAS, bool LSE>
__global__ __launch_bounds__(NT, DB <= 2 ? 3 : 2) void masked_forward(Params p) {
    using T = Tile<DB>;
    constexpr int SLOT = 2 * T::BYTES;  // K, V
    __shared__ __attribute__((aligned(16))) char lds[2 * SLOT];
    __shared__ __attribute__((aligned(16))) int docs[2][TILE];
    __shared__ Spoilt spoilt[NT];
    __shared__ DocRange kept[NW][64];
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int nqb = (p.nq + QB - 1) / QB;
    const Place place = place_in(p.B * p.H, nqb, p.causal, p.kv_doc != nullptr);
    if (place.item < 0) return;
    const int bh = place.item, qb = nqb - 1 - place.block;
    const int b = scalar(bh / p.H), head = bh - b * p.H, kh = scalar(head / p.G);
    const Seq sq = seq_of(p, b);
    const int i0 = qb * QB, last = min(i0 + QB, p.nq) - 1;
    const int w0 = i0 + 32 * wave, wlast = min(w0 + 32, p.nq) - 1;  // the wavefront's queries (w0 > wlast: none)
    const int i = w0 + (lane & 31);
    const bool in = i < p.nq;
    const Row row = row_of(p, sq, b, head, i, in);
    bf16x8 q[2 * DB];
    load_rows<DB>(p.q + b * p.q_batch + (int64_t)min(i, p.nq - 1) * p.q_row + head * p.D, in, p.D, q, lane);

    const int end = tiles_of(limit_of(p, sq, last));
    const int lim_lo = limit_of(p, sq, w0), lim_hi = w0 <= wlast ? limit_of(p, sq, wlast) : 0;
    const int least = limit_of(p, sq, i0);  // every query sees the keys before (documents apart)
    DocWindow window;
    {
        DocRange all = {}, mine = {};
        if (p.kv_doc) {
            mine = range_of_lanes(row.doc, in);
            const DocRange* r = p.q_range + (int64_t)b * tiles_of(p.nq) + i0 / TILE;
            all = r[0];
            if (last / TILE > i0 / TILE) all = joined(all, r[1]);
        }
        window.init(p.kv_range + (int64_t)b * tiles_of(p.nkv), kept[wave], end, all, mine, p.kv_doc != nullptr);
    }

    const Loader<DB, NW, TILE> kload(p.k_row, p.D, wave, lane), vload(p.v_row, p.D, wave, lane);
    const Reader<DB> rd(lane);
    const bf16* kb = p.k + b * p.k_batch + kh * p.D;
    const bf16* vb = p.v + b * p.v_batch + kh * p.D;
    const uint32_t lds0 = lds_address(lds);
    const uint32_t docs0 = lds_address(docs);
    auto issue = [&](int t, int slot) {
        kload.issue(kb, t * TILE, sq.len, lds0 + slot * SLOT);
        vload.issue(vb, t * TILE, sq.len, lds0 + slot * SLOT + T::BYTES);
        if (p.kv_doc && tid < TILE)
            load_lds4(uniform64((uint64_t)(uintptr_t)(p.kv_doc + (int64_t)b * p.nkv + t * TILE)), 4 * min(tid, sq.len - 1 - t * TILE), docs0 + slot * TILE * 4);
    };
    if (2 * p.D < T::RB) {
        clear_tiles(lds, 2 * SLOT, NT);
        __syncthreads();
    }

    spoilt[tid] = Spoilt{0, 0};
    State<DB> st;
    clear(st);
    bool first = true;
    const Context<DB> c = {p, q, row, rd, lane};
    TileOrder order = {-1, end, false};
    if (BIAS && end > 0 && sq.pos0 + last >= 0) order.start = min((sq.pos0 + last) / TILE, end - 1);
    int slot = 0, t;
    bool more = order.first(window, t), same = true, apart = false, same_all = true;
    auto look = [&](int of, bool& a, bool& b_, bool& c_) { a = window.same(of), b_ = window.apart(of), c_ = window.same_all(of); };
    if (more) {
        look(t, same, apart, same_all);
        issue(t, slot);
    }
    while (more) {
        landed();
        __syncthreads();  // the tile is there, and nobody reads the one before any more
        int tn = t;
        bool same_n = true, apart_n = false, same_all_n = true;
        const bool more_n = order.advance(window, tn);
        if (more_n) {
            look(tn, same_n, apart_n, same_all_n);
            issue(tn, slot ^ 1);
        }
        char *kt = lds + slot * SLOT, *vt = kt + T::BYTES;
        if ((t + 1) * TILE > least || !same_all) {
            bool bad = false;
#pragma unroll
            for (int o = 0; o < T::BYTES; o += 16 * NT) bad |= not_finite16(vt + o + 16 * tid);
            if (__syncthreads_or(bad)) {
                for (int h = 0; h < 2; ++h) {
                    const uint32_t seen = keys_seen(p, row, docs[slot] + 32 * h, t * TILE + 32 * h);
                    note_spoilt<DB>(spoilt + tid, vt, 32 * h, spoilt_rows<DB>(vt, 32 * h, seen, lane), seen, lane);
                }
                __syncthreads();
                for (int o = 0; o < T::BYTES; o += 16 * NT) make_finite16(vt + o + 16 * tid);
                __syncthreads();
            }
        }
        const int j0 = t * TILE;
        if (j0 < lim_hi && !apart) {
            step<DB, 2, CAP, BIAS, false, LSE>(c, st, kt, kt + T::BYTES, docs[slot], j0, j0 + TILE > lim_lo || !same, first, []() {});
            first = false;
        }
        t = tn, same = same_n, apart = apart_n, same_all = same_all_n, more = more_n;
        slot ^= 1;
    }
    put_spoilt<DB>(spoilt + tid, st.o);

    const float l = sum_halves(st.l), exact = LSE ? sum_halves(st.exact) : 0.f;
    if (!in) return;
    const float inv = l == 0.f ? 0.f : 1.f / l;
    bf16* out = p.y + b * p.y_batch + (int64_t)i * p.y_row + head * p.D + 4 * (lane >> 5);
#pragma unroll
    for (int mb = 0; mb < DB; ++mb)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            if (32 * mb + 8 * g >= p.D) break;
            bf16x4 v;
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = f32_to_bf16(st.o[mb][4 * g + e] * inv);
            *(bf16x4*)(out + 32 * mb + 8 * g) = v;
        }
    if (LSE && lane < 32) p.lse[(int64_t)bh * p.nq + i] = exact == 0.f ? -INFINITY : (st.m + log2f(exact)) * LN2;
}

// ---- few queries, or few workgroups of many ----
//
// Up to 32 rows (the queries of all heads that share a key head) to a
// workgroup, which takes a piece of the keys; its wavefronts take tiles of 32
// keys in turn, each through LDS tiles of its own without a barrier, two tiles on
// their way, and meet at the end.  Bound by the memory: one token of 8 sequences
// of up to 16384 tokens, 8 key heads of 128, 369 MB in 80 us (4.6 TB/s), and 5
// to join the pieces.  (Keys straight from memory into the operands' registers,
// a row to a lane: 92 us.)

constexpr int FEW_KEYS = 32;

template <int DB, bool CAP, bool BIAS>
__global__ __launch_bounds__(NT, 1) void masked_few(Params p) {
    using T = Tile<DB>;
    constexpr int HALF = FEW_KEYS * T::RB, SLOT = 2 * HALF;
    __shared__ __attribute__((aligned(16))) char lds_all[NW * 2 * SLOT];
    __shared__ __attribute__((aligned(16))) int docs[NW][2][FEW_KEYS];
    __shared__ float ml[NW][32][2];
    __shared__ Spoilt spoilt[NT];
    const int tid = threadIdx.x, lane = tid & 63, col = lane & 31;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int piece = blockIdx.x % p.pieces, rest = blockIdx.x / p.pieces;
    const int rb = rest % p.row_blocks, bk = rest / p.row_blocks;
    const int b = bk / p.KH, kh = bk - b * p.KH;
    const Seq sq = seq_of(p, b);
    const int rows = p.G * p.nq, rho = rb * MASKED_FEW_ROWS + col;
    const bool in = rho < rows;
    const int g = min(rho, rows - 1) / p.nq, i = min(rho, rows - 1) - g * p.nq, head = kh * p.G + g;
    const Row row = row_of(p, sq, b, head, i, true);
    bf16x8 q[2 * DB];
    load_rows<DB>(p.q + b * p.q_batch + (int64_t)i * p.q_row + head * p.D, true, p.D, q, lane);
    DocRange mine = {};
    if (p.kv_doc) mine = range_of_lanes(row.doc, true);
    const DocRange* ranges = p.kv_range + (int64_t)b * tiles_of(p.nkv);
    // the block's queries, of one head, or all
    const int r0 = rb * MASKED_FEW_ROWS, r1 = min(r0 + MASKED_FEW_ROWS, rows) - 1, h0 = r0 / p.nq, h1 = r1 / p.nq;
    const int lim_lo = limit_of(p, sq, h0 == h1 ? r0 - h0 * p.nq : 0), lim_hi = limit_of(p, sq, h0 == h1 ? r1 - h0 * p.nq : p.nq - 1);
    const int tiles = (lim_hi + FEW_KEYS - 1) / FEW_KEYS;
    const int t0 = (int)((int64_t)tiles * piece / p.pieces), t1 = (int)((int64_t)tiles * (piece + 1) / p.pieces);
    char* lds = lds_all + wave * 2 * SLOT;
    const uint32_t lds0 = lds_address(lds);
    using Load = Loader<DB, 1, FEW_KEYS>;
    const Load kload(p.k_row, p.D, 0, lane), vload(p.v_row, p.D, 0, lane);
    const Reader<DB> rd(lane);
    const bf16* kb = p.k + b * p.k_batch + kh * p.D;
    const bf16* vb = p.v + b * p.v_batch + kh * p.D;
    // Every NW-th tile from t down that may hold a document of the rows, 64
    // looked over at a time.  (The queries stand at the end, as a rule, and with
    // a bias by distance the largest scores there too: from there the maximum
    // does not move.)
    int base = 1 << 30;
    uint64_t meets = 0, whole = 0;
    auto next = [&](int t) {
        if (!p.kv_doc) return t;
        while (t >= t0) {
            if (base == 1 << 30 || t <= base - 64 * NW) {
                base = t;
                const int u = t - NW * lane;
                const DocRange r = u >= t0 ? ranges[u / 2] : DocRange{0x7fffffff, -1};
                meets = __ballot(ranges_meet(r, mine));
                whole = __ballot(same_document(r, mine));
            }
            const uint64_t m = meets >> ((base - t) / NW);
            if (m) return t - NW * (int)__builtin_ctzll(m);
            t = base - 64 * NW;
        }
        return t;
    };
    auto same = [&](int t) { return !p.kv_doc || (t >= t0 && (whole >> ((base - t) / NW) & 1)); };
    // Keys and values of two tiles are on their way at a time, each into the
    // place of those just used.
    const uint32_t docs0 = lds_address(docs[wave]);
    auto issue_k = [&](int t, int slot) { kload.issue(kb, t * FEW_KEYS, sq.len, lds0 + slot * SLOT); };
    auto issue_v = [&](int t, int slot) {
        vload.issue(vb, t * FEW_KEYS, sq.len, lds0 + slot * SLOT + HALF);
        if (p.kv_doc && lane < FEW_KEYS)
            load_lds4(uniform64((uint64_t)(uintptr_t)(p.kv_doc + (int64_t)b * p.nkv + t * FEW_KEYS)), 4 * min(lane, sq.len - 1 - t * FEW_KEYS),
                      docs0 + slot * FEW_KEYS * 4);
    };
    if (2 * p.D < T::RB) {
        clear_tiles(lds_all, NW * 2 * SLOT, NT);
        __syncthreads();
    }

    spoilt[tid] = Spoilt{0, 0};
    State<DB> st;
    clear(st);
    bool first = true;
    const Context<DB> c = {p, q, row, rd, lane};
    int slot = 0, t = next(t1 - 1 - wave);
    bool whole_t = same(t), whole_u = false;
    int u = t - NW;  // the tile after t
    if (t >= t0) {
        issue_k(t, 0);
        issue_v(t, 0);
        u = next(u);
        whole_u = same(u);
        if (u >= t0) {
            issue_k(u, 1);
            issue_v(u, 1);
        }
    }
    while (t >= t0) {
        // t's loads, not u's, which were issued after them
        if (u >= t0 && p.kv_doc)
            asm volatile("s_waitcnt vmcnt(%0)" ::"i"(2 * Load::PIECES + 1) : "memory");
        else if (u >= t0)
            asm volatile("s_waitcnt vmcnt(%0)" ::"i"(2 * Load::PIECES) : "memory");
        else
            landed();
        const int j0 = t * FEW_KEYS;
        char *kt = lds + slot * SLOT, *vt = kt + HALF;
        const bool partial = j0 + FEW_KEYS > lim_lo || !whole_t;
        if (partial) {
            bool bad = false;
            for (int o = 0; o < HALF; o += 1024) bad |= not_finite16(vt + o + 16 * lane);
            if (__any(bad)) {
                const uint32_t seen = keys_seen(p, row, docs[wave][slot], j0);
                note_spoilt<DB>(spoilt + tid, vt, 0, spoilt_rows<DB>(vt, 0, seen, lane), seen, lane);
                for (int o = 0; o < HALF; o += 1024) make_finite16(vt + o + 16 * lane);
            }
        }
        const int un = u >= t0 ? next(u - NW) : u;
        const bool whole_n = same(un);
        const bool more = u >= t0 && un >= t0;
        step<DB, 1, CAP, BIAS, true, false>(c, st, kt, vt, docs[wave][slot], j0, partial, first, [&]() {
            if (more) issue_k(un, slot);
        });
        first = false;
        // (the values have been read)
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        if (more) issue_v(un, slot);
        t = u, whole_t = whole_u;
        u = un, whole_u = whole_n;
        slot ^= 1;
    }

    put_spoilt<DB>(spoilt + tid, st.o);

    // The wavefronts' results on one maximum, and their sum.
    const float l = sum_halves(st.l);
    if (lane < 32) {
        ml[wave][col][0] = st.m;
        ml[wave][col][1] = l;
    }
    __syncthreads();
    float m = -INFINITY;
#pragma unroll
    for (int w = 0; w < NW; ++w) m = fmaxf(m, ml[w][col][0]);
    auto factor = [](float mw, float m) { return mw == -INFINITY ? 0.f : mw == m ? 1.f : fast_exp2(mw - m); };
    float total = 0.f;
#pragma unroll
    for (int w = 0; w < NW; ++w) total = __builtin_fmaf(ml[w][col][1], factor(ml[w][col][0], m), total);
    const float f = factor(st.m, m);
    float* o = (float*)lds;  // [register][lane]
    static_assert(DB * 16 * 64 * 4 <= 2 * SLOT, "results in the tiles' place");
#pragma unroll
    for (int mb = 0; mb < DB; ++mb)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[(16 * mb + r) * 64 + lane] = f == 0.f ? 0.f : st.o[mb][r] * f;
    __syncthreads();
    const float inv = total == 0.f ? 0.f : 1.f / total;
#pragma unroll
    for (int u = 0; u < 4 * DB; ++u) {
        const int reg = NW * u + wave;
        float v = 0.f;
#pragma unroll
        for (int w = 0; w < NW; ++w) v += ((const float*)(lds_all + w * 2 * SLOT))[reg * 64 + lane];
        if (p.pieces > 1) {
            p.part_o[((int64_t)blockIdx.x * (16 * DB) + reg) * 64 + lane] = v;
        } else {
            const int c = 32 * (reg >> 4) + 8 * ((reg & 15) >> 2) + 4 * (lane >> 5) + (reg & 3);
            if (in && c < p.D) p.y[b * p.y_batch + (int64_t)i * p.y_row + head * p.D + c] = f32_to_bf16(v * inv);
        }
    }
    if (wave == 0 && lane < 32) {
        if (p.pieces > 1) {
            float* pml = p.part_ml + ((int64_t)blockIdx.x * 32 + col) * 2;
            pml[0] = m;
            pml[1] = total;
        } else if (p.lse && in) {
            p.lse[((int64_t)b * p.H + head) * p.nq + i] = total == 0.f ? -INFINITY : (m + log2f(total)) * LN2;
        }
    }
}

// The pieces of 32 rows joined: a workgroup takes four of the 16 DB registers'
// worth of results.
template <int DB>
__global__ __launch_bounds__(NT) void masked_join(Params p) {
    const int lane = threadIdx.x & 63, col = lane & 31;
    const int part = blockIdx.x % (4 * DB), rest = blockIdx.x / (4 * DB);
    const int reg = 4 * part + (threadIdx.x >> 6);
    const int rb = rest % p.row_blocks, bk = rest / p.row_blocks;
    const int b = bk / p.KH, kh = bk - b * p.KH;
    const float* po = p.part_o + ((int64_t)rest * p.pieces * (16 * DB) + reg) * 64 + lane;
    const float* pml = p.part_ml + ((int64_t)rest * p.pieces * 32 + col) * 2;
    // Eight pieces at a time, all of their loads on their way together.
    float m = -INFINITY, v = 0.f, total = 0.f;
    for (int k0 = 0; k0 < p.pieces; k0 += 8) {
        float mk[8], lk[8], ok[8], top = m;
#pragma unroll
        for (int u = 0; u < 8; ++u) {
            const int k = min(k0 + u, p.pieces - 1);
            mk[u] = pml[(int64_t)k * 64];
            lk[u] = pml[(int64_t)k * 64 + 1];
            ok[u] = po[(int64_t)k * (16 * DB * 64)];
        }
#pragma unroll
        for (int u = 0; u < 8; ++u) {
            if (k0 + u >= p.pieces) mk[u] = -INFINITY;
            top = fmaxf(top, mk[u]);
        }
        const float f = m == top ? 1.f : fast_exp2(m - top);  // (both may be -infinity)
        v *= f;
        total *= f;
#pragma unroll
        for (int u = 0; u < 8; ++u) {
            if (mk[u] == -INFINITY) continue;  // (nothing seen: its sums are 0)
            const float w = mk[u] == top ? 1.f : fast_exp2(mk[u] - top);
            total = __builtin_fmaf(lk[u], w, total);
            v = __builtin_fmaf(ok[u], w, v);
        }
        m = top;
    }
    const int rows = p.G * p.nq, rho = rb * MASKED_FEW_ROWS + col;
    if (rho >= rows) return;
    const int g = rho / p.nq, i = rho - g * p.nq, head = kh * p.G + g;
    const int c = 32 * (reg >> 4) + 8 * ((reg & 15) >> 2) + 4 * (lane >> 5) + (reg & 3);
    if (c < p.D) p.y[b * p.y_batch + (int64_t)i * p.y_row + head * p.D + c] = f32_to_bf16(total == 0.f ? 0.f : v / total);
    if (p.lse && reg == 0 && lane < 32)
        p.lse[((int64_t)b * p.H + head) * p.nq + i] = total == 0.f ? -INFINITY : (m + log2f(total)) * LN2;
}

// Ranges of the documents of 64 tokens each, a wavefront to a tile; the
// queries' tiles first, then the keys'.
__global__ __launch_bounds__(NT) void masked_ranges(Params p) {
    const int lane = threadIdx.x & 63;
    const int nq = tiles_of(p.nq), nkv = tiles_of(p.nkv);
    const int64_t t = (int64_t)blockIdx.x * NW + (threadIdx.x >> 6);
    if (t >= (int64_t)p.B * (nq + nkv)) return;
    const bool keys = t >= (int64_t)p.B * nq;
    const int64_t u = keys ? t - (int64_t)p.B * nq : t;
    const int per = keys ? nkv : nq, n = keys ? p.nkv : p.nq;
    const int b = (int)(u / per), i = (int)(u - (int64_t)b * per) * TILE + lane;
    const int32_t* doc = keys ? p.kv_doc : p.q_doc;
    const DocRange r = range_of_lanes(i < n ? doc[(int64_t)b * n + i] : 0, i < n);
    if (lane == 0) (keys ? p.kv_range : p.q_range)[u] = r;
}

}  // namespace

hipError_t launch_masked_ranges(const Params& p, hipStream_t s) {
    const int64_t t = (int64_t)p.B * (tiles_of(p.nq) + tiles_of(p.nkv));
    masked_ranges<<<(unsigned)((t + NW - 1) / NW), NT, 0, s>>>(p);
    return hipGetLastError();
}

hipError_t launch_masked_forward(const Params& p, hipStream_t s) {
    const int64_t blocks = (int64_t)p.B * p.H * ((p.nq + QB - 1) / QB);
    return with_shape(p, [&](auto db, auto cap, auto bias) {
        if (p.lse)
            masked_forward<db(), cap(), bias(), true><<<blocks_for(blocks), NT, 0, s>>>(p);
        else
            masked_forward<db(), cap(), bias(), false><<<blocks_for(blocks), NT, 0, s>>>(p);
        return hipGetLastError();
    });
}

hipError_t launch_masked_few(const Params& p, hipStream_t s) {
    const int64_t groups = (int64_t)p.B * p.KH * p.row_blocks;
    return with_shape(p, [&](auto db, auto cap, auto bias) {
        masked_few<db(), cap(), bias()><<<(unsigned)(groups * p.pieces), NT, 0, s>>>(p);
        if (p.pieces > 1) {
            const hipError_t e = hipGetLastError();
            if (e != hipSuccess) return e;
            masked_join<db()><<<(unsigned)(groups * 4 * db()), NT, 0, s>>>(p);
        }
        return hipGetLastError();
    });
}

}  // namespace pcpp

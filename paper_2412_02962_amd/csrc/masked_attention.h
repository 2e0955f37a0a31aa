// What the masked attention's kernels share: a call's parameters, the mask,
// the scores' transform and the operands of the matrix products.
//
// A product takes 32 x 32 tiles with the queries or the keys of a wavefront in
// the lanes: of the scores' tile a lane holds one column (lane % 32) and the
// rows 8 (r / 4) + 4 (lane / 32) + r % 4 in register r.  Those registers, eight
// at a time and rounded to bf16, are the second operand of the next product as
// they stand, if its first operand takes the contracted rows in the same order,
// as Reader::columns does.
#pragma once

#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include <type_traits>

#include "common.h"

namespace pcpp {
namespace masked {

constexpr int TILE = 64;             // tokens of a tile of keys or queries
constexpr float LOG2E = 1.4426950408889634f;
constexpr float LN2 = 0.69314718055994531f;

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

// Documents of 64 tokens: the least number, its top bit set where some tokens
// have none, and the largest (-1: all have none).
struct DocRange {
    int32_t lo, hi;
};
constexpr uint32_t SOME_NONE = 0x80000000u;

struct Params {
    const bf16 *q, *k, *v, *dy;
    bf16* y;
    float* lse;                    // [B, H, nq] natural logarithms, or null
    bf16 *dq, *dk, *dv;
    float* delta;                  // [B, H, nq] dy . y, then what masked_dkv adds to dy . v: less the better delta
    float* lse2;                   // [B, H, nq] what it adds to scores: less lse in log2 units
    int64_t q_row, k_row, v_row, y_row, q_batch, k_batch, v_batch, y_batch;
    int32_t B, nq, nkv, H, KH, G;  // G = H / KH query heads to a key head
    int32_t D;                     // channels of a head
    int32_t causal;
    float scale, cap;
    float z_mul;                   // of q . k: into log2 units, or with a cap into the exponent of tanh
    float cap2;                    // cap in log2 units; 0: none
    const int32_t *kv_len, *q_pos, *prefix, *q_doc, *kv_doc;
    const float* slopes;
    DocRange *q_range, *kv_range;  // [B][tiles], with documents
    // few queries: pieces of the keys, their results; keys' gradients: pieces of
    // the queries, [pieces][B * KH][nkv][dk, dv][32 DB] float32 in part_o
    int32_t pieces, row_blocks;
    float* part_o;
    float* part_ml;
};

// Blocks of 32 channels that a head of D is worked in (a tile's rows have 64
// channels at least).
__host__ __device__ inline int blocks_of(int D) { return D <= 64 ? 2 : (D + 31) / 32; }
__host__ __device__ inline int tiles_of(int n) { return (n + TILE - 1) / TILE; }

// Sequence b's keys, first position and prefix.
struct Seq {
    int len, pos0, prefix;
};
__device__ __forceinline__ Seq seq_of(const Params& p, int b) {
    Seq s;
    s.len = p.kv_len ? min(max(p.kv_len[b], 0), p.nkv) : p.nkv;
    s.pos0 = p.q_pos ? min(max(p.q_pos[b], -(1 << 30)), 1 << 30) : p.nkv - p.nq;
    s.prefix = p.prefix ? min(max(p.prefix[b], 0), p.nkv) : 0;
    return s;
}
// Query i sees no key from here on (documents apart).
__device__ __forceinline__ int limit_of(const Params& p, const Seq& s, int i) {
    return p.causal ? min(s.len, max(s.pos0 + i + 1, s.prefix)) : s.len;
}

// Documents of keys are compared as max(number, -1), a query's (of a key's
// workgroup, the key's) as itself or, if it has none, as a number that no key has.
constexpr int NO_DOC = -2;
__device__ __forceinline__ int own_document(int d) { return d >= 0 ? d : NO_DOC; }

__device__ __forceinline__ int least_document(const DocRange& a) { return (int)((uint32_t)a.lo & ~SOME_NONE); }
__device__ __forceinline__ bool ranges_meet(const DocRange& a, const DocRange& b) {
    return a.hi >= least_document(b) && b.hi >= least_document(a);
}
__device__ __forceinline__ bool same_document(const DocRange& a, const DocRange& b) {
    return a.lo >= 0 && a.lo == a.hi && b.lo == a.lo && b.hi == a.lo;
}
__device__ __forceinline__ DocRange joined(const DocRange& a, const DocRange& b) {
    return DocRange{(int)((uint32_t)min(least_document(a), least_document(b)) | (((uint32_t)a.lo | (uint32_t)b.lo) & SOME_NONE)), max(a.hi, b.hi)};
}

// The score of q . k in log2 units before the bias, plus `add`; in `slope` a
// quarter of its derivative by z, (1 - tanh^2) / 4 (without a cap: 1).
// cap tanh(x) = cap - 2 cap / (e^2x + 1): right at both ends without a test,
// off by 2^-23 of the cap in the middle.
template <bool CAP>
__device__ __forceinline__ float score(const Params& p, float dot, float add, float* slope = nullptr) {
    if constexpr (!CAP) {
        if (slope) *slope = 1.f;
        return __builtin_fmaf(dot, p.z_mul, add);
    } else {
        const float r = __builtin_amdgcn_rcpf(fast_exp2(dot * p.z_mul) + 1.f);
        if (slope) *slope = __builtin_fmaf(-r, r, r);
        return __builtin_fmaf(-2.f * p.cap2, r, p.cap2 + add);
    }
}

// ---- tiles in LDS: rows of RB bytes, the channels behind a head's 0.  The 16
// bytes c of row r lie at c ^ swizzle(r).  LDS serves 256 bytes at a time: 16
// rows at one channel (row reads), or four rows of 64 bytes (transposing reads
// by 32 lanes); either lies in different banks.  The swizzle repeats every 16
// rows, and eight rows on it differs in bit 1.  (8192 queries and keys: 34 million
// conflicting cycles with a swizzle by the row's last bits alone, now none.) ----

template <int DB>
struct Tile {
    static constexpr int RB = DB <= 2 ? 128 : 256;  // bytes of a row
    static constexpr int VECS = RB / 16;
    static constexpr int BYTES = TILE * RB;
    __device__ static __forceinline__ int swizzle(int r) {
        if constexpr (RB == 256) return (r & 3) << 2 | (r >> 2 & 3);
        return (r >> 1 & 1) << 2 | (r >> 2 & 3);
    }
};

// 16 bytes per lane from a wave-uniform base and a lane's offset straight into
// LDS, lane l's at lds + 16 l.  In assembly, since the compiler's own tracking
// of such writes would wait for all of them before any LDS read; the kernels
// order them by landed() and barriers.  The base may come out of a vector
// instruction (a lane read) right before: a load may read such a scalar five
// instructions later at the earliest, and within assembly the compiler does not
// see to that.
__device__ __forceinline__ void load_lds(uint64_t base, uint32_t off, uint32_t lds) {
    asm volatile("s_nop 4\n\tglobal_load_lds_dwordx4 %0, %1" ::"v"(off), "s"(base), "{m0}"(lds) : "memory");
}
// The same of 4 bytes, lane l's at lds + 4 l.
__device__ __forceinline__ void load_lds4(uint64_t base, uint32_t off, uint32_t lds) {
    asm volatile("s_nop 4\n\tglobal_load_lds_dword %0, %1" ::"v"(off), "s"(base), "{m0}"(lds) : "memory");
}
__device__ __forceinline__ void landed() { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); }

__device__ __forceinline__ uint64_t uniform64(uint64_t x) {
    const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)x);
    const uint32_t hi = __builtin_amdgcn_readfirstlane((uint32_t)(x >> 32));
    return ((uint64_t)hi << 32) | lo;
}
__device__ __forceinline__ uint32_t lds_address(const void* p) {
    typedef __attribute__((address_space(3))) const void* lptr;
    return __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)(lptr)p);
}

// Tiles of ROWS rows of one tensor: each of NW wavefronts brings its share of
// the rows, 1 KB at a time.  Rows behind the tensor's last are copies of that
// one (their weights are 0).
template <int DB, int NW, int ROWS>
struct Loader {
    using T = Tile<DB>;
    static constexpr int PIECES = ROWS * T::RB / 1024 / NW;
    static constexpr int PIECE_ROWS = 1024 / T::RB;
    static_assert(PIECES >= 1, "shares");
    static constexpr int PERIOD = 16 / PIECE_ROWS;  // pieces until the swizzle repeats
    static constexpr int KINDS = PIECES < PERIOD ? PIECES : PERIOD;
    static_assert(PIECES % KINDS == 0 && (PIECES >= PERIOD ? PIECES % PERIOD == 0 : PERIOD % PIECES == 0), "pieces i and i + KINDS are of a kind");
    uint32_t row_bytes;
    uint32_t off[KINDS];
    int row, first;
    int in;  // bit i: the lane's channels in pieces of kind i are the head's (the others stay 0 in LDS)
    __device__ __forceinline__ Loader(int64_t row_elements, int D, int wave, int lane) {
        row_bytes = (uint32_t)(2 * row_elements);
        row = lane / T::VECS;
        first = PIECES * wave;
        in = 0;
#pragma unroll
        for (int i = 0; i < KINDS; ++i) {
            const int c = (lane % T::VECS) ^ T::swizzle(row + (first + i) * PIECE_ROWS);
            off[i] = (uint32_t)row * row_bytes + 16 * c;
            in |= (8 * c < D) << i;
        }
    }
    // Rows row0 .. of the tensor at `base`, which has `rows`, into the tile at `lds`.
    __device__ __forceinline__ void issue(const bf16* base, int row0, int rows, uint32_t lds) const {
        const uint64_t at = uniform64((uint64_t)(uintptr_t)base + (uint64_t)row0 * row_bytes);
        if (row0 + ROWS <= rows) {
#pragma unroll
            for (int i = 0; i < PIECES; ++i) {
                const int piece = first + i;
                if (in >> (i % KINDS) & 1) load_lds(at + (uint64_t)(piece * PIECE_ROWS) * row_bytes, off[i % KINDS], lds + 1024 * piece);
            }
        } else {
#pragma unroll
            for (int i = 0; i < PIECES; ++i) {
                const int piece = first + i, r = piece * PIECE_ROWS + row, last = rows - 1 - row0;
                const uint32_t o = off[i % KINDS] + (uint32_t)(min(r, last) - row) * row_bytes;
                if (in >> (i % KINDS) & 1) load_lds(at, o, lds + 1024 * piece);
            }
        }
    }
};

// A lane's addresses in a tile (of one slot; the slots' distance is a power of
// two above the tile's bits).
template <int DB>
struct Reader {
    using T = Tile<DB>;
    uint32_t row_at, col_at;
    __device__ __forceinline__ explicit Reader(int lane) {
        const int r = lane & 31;
        row_at = (uint32_t)(r * T::RB + 16 * ((lane >> 5) ^ T::swizzle(r)));
        const int t = 4 * (lane >> 5) + ((lane & 15) >> 2), e = 16 * ((lane >> 4) & 1) + 4 * (lane & 3);
        col_at = (uint32_t)(t * T::RB + 16 * ((e >> 3) ^ T::swizzle(t)) + 2 * (e & 7));
    }
    // The addresses of the reads that follow are worked out there, not kept in
    // registers for the whole loop (TIGHT: where a third wavefront of a SIMD needs
    // them).
    template <bool TIGHT = false>
    __device__ __forceinline__ Reader fresh() const {
        Reader r = *this;
        if constexpr (DB > 2 || TIGHT) asm volatile("" : "+v"(r.row_at), "+v"(r.col_at));
        return r;
    }
    // Rows row0 + (lane % 32), channels 16 kk + 8 (lane / 32) ..: a product
    // that contracts channels.  row0 a multiple of 32.
    __device__ __forceinline__ bf16x8 rows(const char* tile, int row0, int kk) const {
        return *(const bf16x8*)(tile + row0 * T::RB + (row_at ^ (32 * kk)));
    }
    // Channel 32 mb + (lane % 32) of the 16 rows from row0, in the order of the
    // scores' registers: a product that contracts rows.  Two transposing reads
    // of four rows each for either half of the lanes.
    __device__ __forceinline__ bf16x8 columns(const char* tile, int row0, int mb) const {
        typedef short s16x4 __attribute__((ext_vector_type(4)));
        typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
        const char* a = tile + row0 * T::RB;
        const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(a + (col_at ^ (64 * mb))));
        const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(a + 8 * T::RB + (col_at ^ (64 * mb + 32))));
        const short __attribute__((ext_vector_type(8))) w = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
        return __builtin_bit_cast(bf16x8, w);
    }
};

// 0 to the whole of a workgroup's tiles, where a head has fewer channels than
// their rows: what no load writes stays 0, also for the look at infinities and
// NaN, which takes whole rows.
__device__ __forceinline__ void clear_tiles(char* lds, int bytes, int threads) {
    for (int i = 16 * threadIdx.x; i < bytes; i += 16 * threads) *(u32x4*)(lds + i) = u32x4{};
}

// The tiles of a sequence that may hold documents of `all`, 64 looked over at a
// time (a lane each: one by one, each look is a wait for memory), in either
// direction; `mine` is the wavefront's part of `all`.
struct DocWindow {
    const DocRange* ranges;
    DocRange* kept;  // the wavefront's 64 of them, in LDS
    int end, base;
    DocRange all, mine;
    uint64_t meets;
    bool on;
    __device__ __forceinline__ void init(const DocRange* ranges_, DocRange* kept_, int end_, const DocRange& all_, const DocRange& mine_, bool on_) {
        ranges = ranges_, kept = kept_, end = end_, base = -(1 << 30), all = all_, mine = mine_, on = on_;
        meets = 0;
    }
    // The first tile from t on (end: none).
    __device__ __forceinline__ int next(int t) {
        if (!on) return t;
        while (t < end) {
            if (t >= base + TILE || t < base) load(t);
            const uint64_t m = meets >> (t - base);
            if (m) return t + __builtin_ctzll(m);
            t = base + TILE;
        }
        return end;
    }
    // The first tile from t down (-1: none).
    __device__ __forceinline__ int prev(int t) {
        if (!on) return t;
        while (t >= 0) {
            if (t >= base + TILE || t < base) load(t - (TILE - 1));
            const uint64_t m = meets << (TILE - 1 - (t - base));
            if (m) return t - __builtin_clzll(m);
            t = base - 1;
        }
        return -1;
    }
    __device__ __forceinline__ void load(int from) {
        base = from;
        const int u = from + (int)(threadIdx.x & 63);
        const DocRange r = u >= 0 && u < end ? ranges[u] : DocRange{0x7fffffff, -1};
        kept[threadIdx.x & 63] = r;
        meets = __ballot(ranges_meet(r, all));
    }
    // Of a tile that next() has just returned: all of it and of the workgroup,
    // or of the wavefront, one document; none of the wavefront's in it.
    __device__ __forceinline__ DocRange range(int t) const {
        const DocRange r = kept[t - base];
        return DocRange{__builtin_amdgcn_readfirstlane(r.lo), __builtin_amdgcn_readfirstlane(r.hi)};
    }
    __device__ __forceinline__ bool same_all(int t) const { return !on || same_document(range(t), all); }
    __device__ __forceinline__ bool same(int t) const { return !on || same_document(range(t), mine); }
    __device__ __forceinline__ bool apart(int t) const { return on && !ranges_meet(range(t), mine); }
};

// The order of a query block's tiles.  With a bias by distance the scores grow
// towards the queries' own place, and a maximum found on the way there would
// move at every step: from there down first, then from there up.
struct TileOrder {
    int start, end;  // the first tile, or -1: from 0 up only
    bool down;
    __device__ __forceinline__ bool first(DocWindow& w, int& t) {
        down = start >= 0;
        if (down) {
            t = w.prev(start);
            if (t >= 0) return true;
        }
        return turn(w, t);
    }
    __device__ __forceinline__ bool turn(DocWindow& w, int& t) {
        down = false;
        t = w.next(start + 1);
        return t < end;
    }
    // From t to the one after it; false: there is none.
    __device__ __forceinline__ bool advance(DocWindow& w, int& t) {
        if (!down) {
            t = w.next(t + 1);
            return t < end;
        }
        t = w.prev(t - 1);
        return t >= 0 || turn(w, t);
    }
};

// The workgroup's item and block of `items` x `blocks`: neighbours in that list,
// which read the same keys, run on one of the chip's eight parts with a cache of
// their own (workgroup w on part w % 8).  `falling`: an item's blocks grow
// shorter; a part then takes its list by the length, and every other 32
// workgroups backwards, so that its 32 compute units get long and short ones.
// (Forward, before 64 keys a step: 8192 causal queries, 16 heads of 128, 381 us
// item by item with the longest first, 492 with every other item's shortest
// first; 2 x 4096, 10 heads of 64, 149 and 128; this order 350 and 99.)
// `uneven`: documents, the same for all heads, so that blocks of like length come
// at like places: every other 32 workgroups backwards too (2 x 4096, 10 heads,
// 9 documents: forward 74 and 69 us, dq 87 and 82; dk and dv, in two rounds, 110
// and 112: not there).
constexpr int PARTS = 8, PART_UNITS = 32;
// A division's result as the scalar it is.
__device__ __forceinline__ int scalar(int x) { return __builtin_amdgcn_readfirstlane(x); }
struct Place {
    int item, block;  // item < 0: none
};
__device__ __forceinline__ Place place_in(int items, int blocks, bool falling, bool uneven) {
    const int n = items * blocks, per = (n + PARTS - 1) / PARTS;  // (below 2^24)
    const int from = (int)(blockIdx.x % PARTS) * per, to = min(from + per, n);
    const int count = to - from;
    int k = (int)(blockIdx.x / PARTS);
    if (k >= count) return Place{-1, 0};
    const int round = k / PART_UNITS;
    if ((falling || uneven) && (round & 1) && (round + 1) * PART_UNITS <= count) k = round * PART_UNITS + (PART_UNITS - 1 - k % PART_UNITS);
    if (!falling) {
        const int item = scalar((from + k) / blocks);
        return Place{item, from + k - item * blocks};
    }
    // The part's list: item h0 from block o on, whole items, item h1 up to block e.
    const int h0 = scalar(from / blocks), o = from - h0 * blocks;
    const int h1 = scalar(to / blocks), e = to - h1 * blocks;
    if (h0 == h1) return Place{h0, o + k};
    const int head = o > 0, whole = h1 - h0 - head;
    auto before = [&](int block) { return whole * block + (head ? max(block - o, 0) : 0) + min(block, e); };  // blocks of smaller number
    int lo = 0, hi = blocks - 1;  // the largest with before() <= k
    while (lo < hi) {
        const int mid = (lo + hi + 1) / 2;
        if (before(mid) <= k)
            lo = mid;
        else
            hi = mid - 1;
    }
    const int skip = head && lo < o;
    return Place{h0 + skip + k - before(lo), lo};
}
inline unsigned blocks_for(int64_t n) { return (unsigned)((n + PARTS - 1) / PARTS * PARTS); }

// Rows of a tensor as the second operand of a product over channels: row
// (lane % 32), zeros where there is none.
template <int DB>
__device__ __forceinline__ void load_rows(const bf16* row, bool in, int D, bf16x8 (&o)[2 * DB], int lane) {
#pragma unroll
    for (int kk = 0; kk < 2 * DB; ++kk) {
        const int c = 16 * kk + 8 * (lane >> 5);
        o[kk] = in && c < D ? *(const bf16x8*)(row + c) : bf16x8{};
    }
}

// Sixteen registers as two operands.
__device__ __forceinline__ void pack(const float (&w)[16], bf16x8 (&o)[2]) {
#pragma unroll
    for (int r = 0; r < 16; ++r) o[r >> 3][r & 7] = f32_to_bf16(w[r]);
}

// use(i, read(i)) for i = 0 .. N - 1, the reads AHEAD of their uses: where the
// registers are few, the compiler's own order is each read, its wait, its use
// (8192 causal, heads of 128, us: forward 315 and 304 with two ahead, dq 432 and
// 425, dk and dv 645 and 609; one, three and four ahead are within 1 % of that).
template <int N, int AHEAD, typename Read, typename Use>
__device__ __forceinline__ void staged(Read read, Use use) {
    decltype(read(0)) ring[AHEAD + 1];
#pragma unroll
    for (int i = 0; i < AHEAD && i < N; ++i) ring[i] = read(i);
#pragma unroll
    for (int i = 0; i < N; ++i) {
        if (i + AHEAD < N) ring[(i + AHEAD) % (AHEAD + 1)] = read(i + AHEAD);
        __builtin_amdgcn_sched_barrier(0);
        use(i, ring[i % (AHEAD + 1)]);
    }
}

// acc += sum over 32 HB rows from row0 of (their weights) x (their channels).
template <int DB, int HB>
__device__ __forceinline__ void add_rows(f32x16 (&acc)[DB], const bf16x8 (&w)[HB][2], const Reader<DB>& rd, const char* tile, int row0) {
    staged<2 * DB * HB, 2>([&](int i) __attribute__((always_inline)) { return rd.columns(tile, row0 + 16 * (i / DB), i % DB); },
                               [&](int i, const bf16x8& x) __attribute__((always_inline)) {
                                   const int st = i / DB, mb = i % DB;
                                   acc[mb] = mfma32x32x16(x, w[st >> 1][st & 1], acc[mb]);
                               });
}

// ---- infinities and NaN in rows that the mask hides from some lanes ----
//
// A product over rows takes 0 x infinity from a row that a lane's weight of 0
// hides.  So a tile that some lane does not see all of is looked over when it has
// landed; where it holds infinities or NaN (never, in a sound program), every
// lane notes which of its sums they belong to, and which of its scores they make
// infinite or NaN where these are products with the same tile; then they become 0
// in LDS.

// Sixteen bytes at a: whether there are any; and 0 in their place.
__device__ __forceinline__ bool not_finite16(const char* a) {
    const u32x4 w = *(const u32x4*)a;
    bool bad = false;
#pragma unroll
    for (int e = 0; e < 4; ++e) bad |= (w[e] & 0x7f80u) == 0x7f80u || (w[e] & 0x7f800000u) == 0x7f800000u;
    return bad;
}
__device__ __forceinline__ void make_finite16(char* a) {
    u32x4 w = *(const u32x4*)a;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        if ((w[e] & 0x7f80u) == 0x7f80u) w[e] &= 0xffff0000u;
        if ((w[e] & 0x7f800000u) == 0x7f800000u) w[e] &= 0x0000ffffu;
    }
    *(u32x4*)a = w;
}

// Which of a lane's sums take an infinity of either sign (NaN: both): a bit for
// each, in LDS, so that the products' loop has the registers.
struct Spoilt {
    uint64_t plus, minus;
};
// Which of the 32 rows from row0 of a tile have any (a bit each), if some lane
// sees such a row, `seen` its rows; else 0: nobody's sums and scores take any.
template <int DB>
__device__ __forceinline__ uint32_t spoilt_rows(const char* tile, int row0, uint32_t seen, int lane) {
    bool bad = false;
#pragma unroll 1
    for (int c = lane >> 5; c < Tile<DB>::VECS; c += 2) bad |= not_finite16(tile + (row0 + (lane & 31)) * Tile<DB>::RB + 16 * c);
    const uint64_t both = __ballot(bad);
    const uint32_t rows = (uint32_t)both | (uint32_t)(both >> 32);
    return __any((seen & rows) != 0) ? rows : 0u;
}
// Those rows of a tile; bit j of `seen`: the lane sees row j.
template <int DB>
__device__ __forceinline__ void note_spoilt(Spoilt* mine, const char* tile, int row0, uint32_t rows, uint32_t seen, int lane) {
    uint64_t plus = mine->plus, minus = mine->minus;
#pragma unroll 1
    for (; rows; rows &= rows - 1) {
        const int j = __builtin_ctz(rows);
        const bool sees = seen >> j & 1;
#pragma unroll 1
        for (int g = 0; g < 4 * DB; ++g) {
            const int at = (row0 + j) * Tile<DB>::RB + 16 * (g ^ Tile<DB>::swizzle(j)) + 8 * (lane >> 5);
            const u32x2 w = *(const u32x2*)(tile + at);
            uint32_t up = 0, down = 0;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const uint32_t h = w[e >> 1] >> (16 * (e & 1)) & 0xffffu;
                const bool nan = (h & 0x7fffu) > 0x7f80u;
                up |= (uint32_t)(sees & (nan | (h == 0x7f80u))) << e;
                down |= (uint32_t)(sees & (nan | (h == 0xff80u))) << e;
            }
            plus |= (uint64_t)up << (4 * g);
            minus |= (uint64_t)down << (4 * g);
        }
    }
    mine->plus = plus;
    mine->minus = minus;
}
// Into the sums: with weights above 0 an infinity stays one; `no_number`: with
// weights of 0 it is NaN.
template <int DB>
__device__ __forceinline__ void put_spoilt(const Spoilt* mine, f32x16 (&acc)[DB], bool no_number = false) {
    uint64_t plus = mine->plus, minus = mine->minus;
    if (!__any((plus | minus) != 0)) return;
    if (no_number) plus = minus = plus | minus;
#pragma unroll
    for (int mb = 0; mb < DB; ++mb)
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            if (plus >> (16 * mb + r) & 1) acc[mb][r] += INFINITY;
            if (minus >> (16 * mb + r) & 1) acc[mb][r] -= INFINITY;
        }
}

// What those rows make of the lane's scores with them, `own` its own row in
// memory: bit r for infinity in register r, bit 16 + r for -infinity, both for
// NaN.  (One by one: a product of matrices in this place would cost the kernels
// 25 registers more.)
template <int DB>
__device__ __forceinline__ uint32_t note_scores(const char* tile, int row0, uint32_t rows, const bf16* own, int D, int lane) {
    uint32_t odd = 0;
#pragma unroll 1
    for (; rows; rows &= rows - 1) {
        const int j = __builtin_ctz(rows), r = 4 * (j >> 3) + (j & 3);
        if ((j >> 2 & 1) != lane >> 5) continue;
        float z = 0.f;
#pragma unroll 1
        for (int g = 0; g < D / 8; ++g) {
            const char* at = tile + (row0 + j) * Tile<DB>::RB + 16 * (g ^ Tile<DB>::swizzle(j));
            if (!not_finite16(at)) continue;
#pragma unroll 1
            for (int e = 0; e < 8; ++e) {
                const float x = bf16_to_f32(((const bf16*)at)[e]);
                if (!(fabsf(x) < INFINITY)) z = __builtin_fmaf(x, bf16_to_f32(own[8 * g + e]), z);
            }
        }
        odd |= (uint32_t)!(z < INFINITY) << r | (uint32_t)!(z > -INFINITY) << (16 + r);
    }
    return odd;
}
// What the product with the cleaned rows is added to.
__device__ __forceinline__ void put_scores(uint32_t odd, f32x16& s) {
#pragma unroll
    for (int r = 0; r < 16; ++r) {
        s[r] += (odd >> r & 1 ? INFINITY : 0.f) - (odd >> (16 + r) & 1 ? INFINITY : 0.f);
        asm volatile("" : "+v"(odd));
    }
}

__device__ __forceinline__ float max_halves(float v) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float sum_halves(float v) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// The documents of a wavefront's lanes, those that are `in`.
__device__ __forceinline__ DocRange range_of_lanes(int doc, bool in) {
    int lo = in && doc >= 0 ? doc : 0x7fffffff, hi = in ? max(doc, -1) : -1;
    const bool none = __any(in && doc < 0);
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) {
        lo = min(lo, __shfl_xor(lo, d));
        hi = max(hi, __shfl_xor(hi, d));
    }
    lo = __builtin_amdgcn_readfirstlane(lo);
    return DocRange{(int)((uint32_t)lo | (none ? SOME_NONE : 0u)), __builtin_amdgcn_readfirstlane(hi)};
}

}  // namespace masked

// The launches, all asynchronous on s.
hipError_t launch_masked_ranges(const masked::Params& p, hipStream_t s);
hipError_t launch_masked_forward(const masked::Params& p, hipStream_t s);
hipError_t launch_masked_few(const masked::Params& p, hipStream_t s);  // p.pieces, p.row_blocks set
hipError_t launch_masked_delta(const masked::Params& p, hipStream_t s);
hipError_t launch_masked_dq(const masked::Params& p, hipStream_t s);
hipError_t launch_masked_dkv(const masked::Params& p, hipStream_t s);

constexpr int MASKED_FEW_ROWS = 32;  // rows (queries x heads of a key head) of a workgroup of launch_masked_few

// f(head's channels in blocks of 32, capped, biased).  Capped scores without a
// bias take the biased form with slopes of 0: two operations of a dozen more.
template <typename F>
hipError_t with_shape(const masked::Params& p, F f) {
    using std::integral_constant;
    using std::bool_constant;
    auto variant = [&](auto db) {
        if (p.cap2 != 0.f) return f(db, bool_constant<true>(), bool_constant<true>());
        return p.slopes ? f(db, bool_constant<false>(), bool_constant<true>()) : f(db, bool_constant<false>(), bool_constant<false>());
    };
    switch (masked::blocks_of(p.D)) {
        case 2: return variant(integral_constant<int, 2>());
        case 3: return variant(integral_constant<int, 3>());
        default: return variant(integral_constant<int, 4>());
    }
}

}  // namespace pcpp

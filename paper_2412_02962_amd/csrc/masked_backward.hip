// Masked attention, backward: the gradient of the queries (masked_dq, a block
// of queries against all keys) and of keys and values (masked_dkv, a block of
// keys against the queries of all heads that read them), each computing the
// scores again.  Two kernels that own what they write, and so no atomics, for
// two more products than one that adds to dq from everywhere.  See
// masked_attention.h for the operands' layout.

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

template <int DB>
__global__ __launch_bounds__(NT, DB > 3 ? 1 : 2) void masked_dq(Params p) {
    using T = Tile<DB>;
    __shared__ __attribute__((aligned(16))) char kt[T::BYTES], vt[T::BYTES];
    __shared__ __attribute__((aligned(16))) int docs[TILE];
    __shared__ int redo;
    const int tid = threadIdx.x, lane = tid & 63, half = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int nqb = (p.nq + BLOCK - 1) / BLOCK;
    const int bh = blockIdx.x / nqb, qb = blockIdx.x - bh * nqb;
    const int b = bh / p.H, head = bh - b * p.H, kh = head / p.G;
    const Seq sq = seq_of(p, b);
    const int i0 = qb * BLOCK, last = min(i0 + BLOCK, p.nq) - 1;
    const int w0 = i0 + 32 * wave, wlast = min(w0 + 32, p.nq) - 1;
    const int i = w0 + (lane & 31), ic = min(i, p.nq - 1);
    const bool in = i < p.nq;
    const int pos = sq.pos0 + i, limit = limit_of(p, sq, i);
    const int doc = in && p.q_doc ? p.q_doc[(int64_t)b * p.nq + i] : -1;
    const float slope2 = p.slopes ? p.slopes[head] * LOG2E : 0.f;
    const float lse2 = p.lse[(int64_t)bh * p.nq + ic] * LOG2E, delta = p.delta[(int64_t)bh * p.nq + ic];
    bf16x8 q[2 * DB], dy[2 * DB];
    load_rows<DB>(p.q + b * p.q_batch + (int64_t)ic * p.q_row + head * p.D, in, p.D, q, lane);
    load_rows<DB>(p.dy + b * p.y_batch + (int64_t)ic * p.y_row + head * p.D, in, p.D, dy, lane);

    DocRange all = {}, mine = {};
    if (p.kv_doc) {
        mine = range_of_lanes(doc, in);
        const DocRange* r = p.q_range + (int64_t)b * tiles_of(p.nq) + i0 / TILE;
        all = r[0];
        if (last / TILE > i0 / TILE) all = DocRange{min(all.lo, r[1].lo), max(all.hi, r[1].hi)};
    }
    const DocRange* ranges = p.kv_range + (int64_t)b * tiles_of(p.nkv);
    const int end = tiles_of(limit_of(p, sq, last));
    const int lim_lo = limit_of(p, sq, w0), lim_hi = w0 <= wlast ? limit_of(p, sq, wlast) : 0;
    auto next = [&](int t) {
        if (p.kv_doc)
            while (t < end && !ranges_meet(ranges[t], all)) ++t;
        return t;
    };
    u32x4 kr[DB], vr[DB];
    int dr = -1;
    const bf16* kb = p.k + b * p.k_batch + kh * p.D;
    const bf16* vb = p.v + b * p.v_batch + kh * p.D;
    auto load = [&](int t) {
#pragma unroll
        for (int u = 0; u < DB; ++u) {
            const int id = tid + NT * u, r = id / T::VECS, c = 8 * (id - r * T::VECS);
            const int j = t * TILE + r;
            const bool ok = j < sq.len && c < p.D;
            kr[u] = ok ? *(const u32x4*)(kb + j * p.k_row + c) : u32x4{};
            vr[u] = ok ? *(const u32x4*)(vb + j * p.v_row + c) : u32x4{};
        }
        if (p.kv_doc && tid < TILE) dr = t * TILE + tid < sq.len ? p.kv_doc[(int64_t)b * p.nkv + t * TILE + tid] : -1;
    };
    auto store = [&]() {
#pragma unroll
        for (int u = 0; u < DB; ++u) {
            const int id = tid + NT * u, r = id / T::VECS, c = id - r * T::VECS;
            *(u32x4*)(kt + r * T::LD + 16 * c) = kr[u];
            *(u32x4*)(vt + r * T::LD + 16 * c) = vr[u];
        }
        if (p.kv_doc && tid < TILE) docs[tid] = dr;
    };

    f32x16 acc[DB];
    auto step = [&](int row0, int j0, bool partial, bool careful) __attribute__((always_inline)) {
        f32x16 s, dp;
#pragma unroll
        for (int kk = 0; kk < 2 * DB; ++kk) {
            s = mfma32x32x16(row_operand<DB>(kt, row0, kk, lane), q[kk], kk == 0 ? f32x16{} : s);
            dp = mfma32x32x16(row_operand<DB>(vt, row0, kk, lane), dy[kk], kk == 0 ? f32x16{} : dp);
        }
        float w[16];
        const int base = j0 + 4 * half;
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            i32x4 d = {};
            if (partial && p.kv_doc) d = *(const i32x4*)(docs + row0 + 8 * g + 4 * half);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int r = 4 * g + e;
                float sl, x = score(p, s[r], &sl);
                if (slope2 != 0.f) x = __builtin_fmaf(-slope2, (float)abs(pos - base - (8 * g + e)), x);
                const float pr = fast_exp2(x - lse2);
                const bool seen = !partial || (base + 8 * g + e < limit && (!p.kv_doc || (d[e] == doc && d[e] >= 0)));
                w[r] = seen ? pr * (dp[r] - delta) * sl : 0.f;
            }
        }
        if (careful && partial)
            add_rows_careful<DB>(acc, w, kt, row0, lane);
        else
            add_rows<DB>(acc, w, kt, row0, lane);
    };

    for (int pass = 0; pass < 2; ++pass) {
        clear<DB>(acc);
        int t = next(0);
        if (t < end) load(t);
        while (t < end) {
            __syncthreads();
            store();
            __syncthreads();
            const int tn = next(t + 1);
            if (tn < end) load(tn);
#pragma unroll 1
            for (int h = 0; h < 2; ++h) {
                const int j0 = t * TILE + 32 * h;
                if (j0 >= lim_hi) continue;
                step(32 * h, j0, j0 + 32 > lim_lo || (p.kv_doc && !same_document(ranges[t], mine)), pass > 0);
            }
            t = tn;
        }
        if (pass > 0) break;
        __syncthreads();
        if (tid == 0) redo = 0;
        __syncthreads();
        if (any_not_finite<DB>(acc) && lane == 0) redo = 1;
        __syncthreads();
        if (!redo) break;
    }
    if (in) store_rows<DB>(p.dq + b * p.q_batch + (int64_t)i * p.q_row + head * p.D, acc, p.scale, p.D, lane);
}

// What a tile's queries bring besides q and dy.
struct QueryTile {
    float lse2[TILE], delta[TILE];
    int limit[TILE], doc[TILE];
};

template <int DB>
__global__ __launch_bounds__(NT, 1) void masked_dkv(Params p) {
    using T = Tile<DB>;
    __shared__ __attribute__((aligned(16))) char qt[T::BYTES], gt[T::BYTES];
    __shared__ __attribute__((aligned(16))) QueryTile rows;
    __shared__ int redo;
    const int tid = threadIdx.x, lane = tid & 63, half = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int nkb = (p.nkv + BLOCK - 1) / BLOCK;
    const int bk = blockIdx.x / nkb, kb = blockIdx.x - bk * nkb;
    const int b = bk / p.KH, kh = bk - b * p.KH;
    const Seq sq = seq_of(p, b);
    const int k0 = kb * BLOCK, klast = min(k0 + BLOCK, p.nkv) - 1;
    const int w0 = k0 + 32 * wave;
    const int j = w0 + (lane & 31);
    const bool in = j < p.nkv, live = j < sq.len;
    const int doc = live && p.kv_doc ? p.kv_doc[(int64_t)b * p.nkv + j] : -1;
    bf16x8 k[2 * DB], v[2 * DB];
    load_rows<DB>(p.k + b * p.k_batch + (int64_t)min(j, p.nkv - 1) * p.k_row + kh * p.D, live, p.D, k, lane);
    load_rows<DB>(p.v + b * p.v_batch + (int64_t)min(j, p.nkv - 1) * p.v_row + kh * p.D, live, p.D, v, lane);

    DocRange all = {}, mine = {};
    if (p.kv_doc) {
        mine = range_of_lanes(doc, live);
        const DocRange* r = p.kv_range + (int64_t)b * tiles_of(p.nkv) + k0 / TILE;
        all = r[0];
        if (klast / TILE > k0 / TILE) all = DocRange{min(all.lo, r[1].lo), max(all.hi, r[1].hi)};
    }
    const DocRange* ranges = p.q_range + (int64_t)b * tiles_of(p.nq);
    // The queries' limits grow: from the first that sees the block's first key.
    const int ntq = tiles_of(p.nq);
    int first = 0;
    if (p.causal && k0 >= sq.prefix) first = min(max(k0 - sq.pos0, 0), p.nq) / TILE;
    if (k0 >= sq.len) first = ntq;
    const int tiles = ntq - min(first, ntq);  // of each head
    const int steps = tiles * p.G;
    auto next = [&](int t) {
        if (p.kv_doc)
            while (t < steps && !ranges_meet(ranges[first + t % tiles], all)) ++t;
        return t;
    };
    u32x4 qr[DB], gr[DB];
    float lr = 0.f, er = 0.f;
    int mr = 0, dr = -1;
    auto load = [&](int t) {
        const int g = t / tiles, i0 = (first + t - g * tiles) * TILE, head = kh * p.G + g;
        const bf16* qb = p.q + b * p.q_batch + head * p.D;
        const bf16* gb = p.dy + b * p.y_batch + head * p.D;
#pragma unroll
        for (int u = 0; u < DB; ++u) {
            const int id = tid + NT * u, r = id / T::VECS, c = 8 * (id - r * T::VECS);
            const int i = i0 + r;
            const bool ok = i < p.nq && c < p.D;
            qr[u] = ok ? *(const u32x4*)(qb + i * p.q_row + c) : u32x4{};
            gr[u] = ok ? *(const u32x4*)(gb + i * p.y_row + c) : u32x4{};
        }
        if (tid < TILE) {
            const int i = i0 + tid;
            const bool ok = i < p.nq;
            const int64_t at = ((int64_t)b * p.H + head) * p.nq + i;
            lr = ok ? p.lse[at] * LOG2E : 0.f;
            er = ok ? p.delta[at] : 0.f;
            mr = ok ? limit_of(p, sq, i) : 0;
            dr = ok && p.q_doc ? p.q_doc[(int64_t)b * p.nq + i] : -1;
        }
    };
    auto store = [&]() {
#pragma unroll
        for (int u = 0; u < DB; ++u) {
            const int id = tid + NT * u, r = id / T::VECS, c = id - r * T::VECS;
            *(u32x4*)(qt + r * T::LD + 16 * c) = qr[u];
            *(u32x4*)(gt + r * T::LD + 16 * c) = gr[u];
        }
        if (tid < TILE) {
            rows.lse2[tid] = lr;
            rows.delta[tid] = er;
            rows.limit[tid] = mr;
            rows.doc[tid] = dr;
        }
    };

    f32x16 dk[DB], dv[DB];
    auto step = [&](int row0, int i0, float slope2, bool partial, bool careful) __attribute__((always_inline)) {
        f32x16 s, dp;
#pragma unroll
        for (int kk = 0; kk < 2 * DB; ++kk) {
            s = mfma32x32x16(row_operand<DB>(qt, row0, kk, lane), k[kk], kk == 0 ? f32x16{} : s);
            dp = mfma32x32x16(row_operand<DB>(gt, row0, kk, lane), v[kk], kk == 0 ? f32x16{} : dp);
        }
        float w[16], z[16];
        const int d0 = sq.pos0 + i0 + 4 * half - j;
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            const int at = row0 + 8 * g + 4 * half;
            const f32x4 lse2 = *(const f32x4*)(rows.lse2 + at), delta = *(const f32x4*)(rows.delta + at);
            i32x4 lim = {}, d = {};
            if (partial) {
                lim = *(const i32x4*)(rows.limit + at);
                d = *(const i32x4*)(rows.doc + at);
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int r = 4 * g + e;
                float sl, x = score(p, s[r], &sl);
                if (slope2 != 0.f) x = __builtin_fmaf(-slope2, (float)abs(d0 + 8 * g + e), x);
                const bool seen = !partial || (j < lim[e] && (!p.kv_doc || (d[e] == doc && d[e] >= 0)));
                const float pr = fast_exp2(x - lse2[e]);
                w[r] = seen ? pr : 0.f;
                z[r] = seen ? pr * (dp[r] - delta[e]) * sl : 0.f;
            }
        }
        if (careful && partial) {
            add_rows_careful<DB>(dv, w, gt, row0, lane);
            add_rows_careful<DB>(dk, z, qt, row0, lane);
        } else {
            add_rows<DB>(dv, w, gt, row0, lane);
            add_rows<DB>(dk, z, qt, row0, lane);
        }
    };

    for (int pass = 0; pass < 2; ++pass) {
        clear<DB>(dk);
        clear<DB>(dv);
        int t = next(0);
        if (t < steps) load(t);
        while (t < steps) {
            __syncthreads();
            store();
            __syncthreads();
            const int tn = next(t + 1);
            if (tn < steps) load(tn);
            const int g = t / tiles, tile = first + t - g * tiles;
            const float slope2 = p.slopes ? p.slopes[kh * p.G + g] * LOG2E : 0.f;
#pragma unroll 1
            for (int h = 0; h < 2; ++h) {
                const int i0 = tile * TILE + 32 * h;
                if (i0 >= p.nq || w0 >= limit_of(p, sq, min(i0 + 31, p.nq - 1))) continue;
                const bool partial = i0 + 32 > p.nq || w0 + 32 > limit_of(p, sq, i0) ||
                                     (p.kv_doc && !same_document(ranges[tile], mine));
                step(32 * h, i0, slope2, partial, pass > 0);
            }
            t = tn;
        }
        if (pass > 0) break;
        __syncthreads();
        if (tid == 0) redo = 0;
        __syncthreads();
        if ((any_not_finite<DB>(dk) || any_not_finite<DB>(dv)) && lane == 0) redo = 1;
        __syncthreads();
        if (!redo) break;
    }
    if (!in) return;
    store_rows<DB>(p.dk + b * p.k_batch + (int64_t)j * p.k_row + kh * p.D, dk, p.scale, p.D, lane);
    store_rows<DB>(p.dv + b * p.v_batch + (int64_t)j * p.v_row + kh * p.D, dv, 1.f, p.D, lane);
}

}  // namespace

hipError_t launch_masked_delta(const Params& p, hipStream_t s) {
    const int64_t rows = (int64_t)p.B * p.nq * p.H;
    masked_delta<<<(unsigned)((rows + NT / 16 - 1) / (NT / 16)), NT, 0, s>>>(p);
    return hipGetLastError();
}

hipError_t launch_masked_dq(const Params& p, hipStream_t s) {
    const int64_t blocks = (int64_t)p.B * p.H * ((p.nq + BLOCK - 1) / BLOCK);
    return with_blocks(p.D, [&](auto db) {
        masked_dq<db()><<<(unsigned)blocks, NT, 0, s>>>(p);
        return hipGetLastError();
    });
}

hipError_t launch_masked_dkv(const Params& p, hipStream_t s) {
    const int64_t blocks = (int64_t)p.B * p.KH * ((p.nkv + BLOCK - 1) / BLOCK);
    return with_blocks(p.D, [&](auto db) {
        masked_dkv<db()><<<(unsigned)blocks, NT, 0, s>>>(p);
        return hipGetLastError();
    });
}

}  // namespace pcpp

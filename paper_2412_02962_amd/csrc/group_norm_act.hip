// GroupNorm with its activation and dropout on channels-last rows, for
// training (and inference in float32 or with GELU), and its backward pass.
//   pcpp_group_norm_act           n = (x - mean) rstd;  z = n gamma + beta;
//                                 y = dropped(act(z))
//   pcpp_group_norm_act_backward  g = dropped(dy) act'(z);  w = g gamma;
//                                 dx = rstd (w - mean(w) - n mean(w n));
//                                 dgamma = sum g n;  dbeta = sum g
//
// Both directions are bound by the memory, in two launches each: sums over a
// chunk of tokens and a slab of channels (whole groups, whole vectors of
// eight) into a record per chunk and group; then the rows again, with the
// records merged by every workgroup that needs them.  A thread keeps its eight
// channels for all of its rows, so that their parameters stay in registers.
// Nothing of the forward pass but mean and rstd is kept: z, the activation's
// derivative and dropout's mask are computed again.  Few tokens take one launch,
// a slab of an image in a workgroup's registers (whole_of).
//
// 2 x 57600 x 640 bf16, SiLU, dropout: statistics 40 us (3.7 TB/s), apply 66
// (4.5), sums 77 (3.8; the vector unit's: the mask and the activation), dx 86
// (5.1), and 5 for each merging of records; 2 x 65536 x 320 without dropout 23,
// 5 and 28.  The rows of a thread are on their way ROWS at a time while as many
// are worked on (without that forward and backward 316 us, with it 280).

#include <stdint.h>

#include "../../include/pcpp.h"
#include "args.h"
#include "common.h"
#include "dropout.h"
#include "ff_act.h"
#include "gemm.h"
#include "rows8.h"

#define PCPP_EXPORT extern "C" __attribute__((visibility("default")))

namespace pcpp {

namespace {

constexpr int kMaxThreads = 512;
constexpr int kMaxTokens = 1 << 30;  // row numbers are 32 bits, those of rows on their way behind the last too
constexpr int kMaxGroups = 256;
constexpr int kRunRows = 8;      // rows that a thread of the statistics takes at a time
constexpr int kBlocks = 512;     // workgroups of a launch that sums: two to a compute unit
// A slab of an image in a workgroup's registers: the rows that a thread holds,
// and, where the slab has several groups, half as many (see whole_of).
constexpr int kWholeRows = 8, kGradRows = 6;
constexpr int kWholeBlocks = 256;
constexpr int kWholeVectors = 4; // of such a slab's rows, at least
constexpr int kFewChunks = 32;   // chunks whose records every consumer merges; more are merged in a launch of their own

// How a launch cuts [B, N, C]: slabs of S channels (whole groups), chunks of
// tokens; a thread holds one vector of V in a row, RP rows side by side.
struct Cut {
    int32_t B, N, C, G;
    int32_t cg;       // channels of a group
    int32_t S, V, RP, gs;
    int32_t chunks;   // of the launch that sums
    int32_t threads;
};

struct NormActParams {
    const void* x;
    const void* dy;      // backward
    const bf16* gamma;
    const bf16* beta;
    void* y;             // forward's y, backward's dx
    float* stats;        // [B][G][2] mean, rstd: forward writes it (or null), backward reads it
    float* records;      // forward [B][chunks][G][3] count, mean, M2; backward [B][chunks][G][2] sums of w, w n
    float* merged;       // the records of all chunks as one, or null: `records` are few
    float* columns;      // backward: [2][B * chunks][C] sums of g n and g, or null
    bf16* dgamma;
    bf16* dbeta;
    Dropout drop;
    Cut cut;
    int32_t apply_blocks;  // workgroups of the apply launch that apply, per slab and image
    float eps;
};

// Eight channels as they lie in memory, so that rows on their way take few
// registers.
template <typename T>
struct Raw;
template <>
struct Raw<bf16> {
    bf16x8 a;
    __device__ __forceinline__ void load(const bf16* p) { a = *(const bf16x8*)p; }
    __device__ __forceinline__ void get(float (&v)[8]) const {
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = bf16_to_f32(a[e]);
    }
};
template <>
struct Raw<float> {
    f32x4 a, b;
    __device__ __forceinline__ void load(const float* p) {
        a = *(const f32x4*)p;
        b = *(const f32x4*)(p + 4);
    }
    __device__ __forceinline__ void get(float (&v)[8]) const {
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = a[e], v[4 + e] = b[e];
    }
};

// A thread's rows t, t + RP, .. of a tensor, ROWS at a time, the next ROWS on
// their way while these are worked on.
template <typename T, int ROWS>
struct Rows {
    Raw<T> cur[ROWS], next[ROWS];
    __device__ __forceinline__ static void fetch(Raw<T> (&to)[ROWS], const T* base, int t, int hi, const Cut& a) {
#pragma unroll
        for (int i = 0; i < ROWS; ++i)
            if (t + i * a.RP < hi) to[i].load(base + (int64_t)(t + i * a.RP) * a.C);
    }
    __device__ __forceinline__ void begin(const T* base, int t, int hi, const Cut& a) { fetch(cur, base, t, hi, a); }
    __device__ __forceinline__ void ahead(const T* base, int t, int hi, const Cut& a) { fetch(next, base, t + ROWS * a.RP, hi, a); }
    __device__ __forceinline__ void step() {
#pragma unroll
        for (int i = 0; i < ROWS; ++i) cur[i] = next[i];
    }
};

// c / cg without a division, by the inverse: exact for c below 2^13.
__device__ __forceinline__ int group_of(int c, float inv_cg) { return (int)(((float)c + 0.5f) * inv_cg); }

// Row lane, vector and channel of a thread; false for the threads left over.
struct Place {
    int r, v, c0;
    bool in;
};
__device__ __forceinline__ Place place_of(const Cut& a, int slab) {
    const int r = group_of(threadIdx.x, 1.f / (float)a.V), v = threadIdx.x - r * a.V;
    return Place{r, v, slab * a.S + 8 * v, r < a.RP};
}

// The sum of v over T consecutive lanes (a power of two up to a wavefront), in
// each of them.
__device__ __forceinline__ float lanes_sum(float v, int T) {
    for (int d = 1; d < T; d <<= 1) v += __shfl_xor(v, d);
    return v;
}
// Lanes that share a group of the slab.
__device__ __forceinline__ int group_lanes(int threads, int gs) {
    int t = 1;
    while (2 * t * gs <= threads && t < 64) t *= 2;
    return t;
}

// ---- statistics ----

// A thread's rows in runs of ROWS, each with its own mean and squared
// deviations (two passes over registers), merged into the thread's by Chan et
// al.'s update: no difference of large sums anywhere.
template <typename T, int ROWS>
__global__ __launch_bounds__(kMaxThreads) void norm_act_stats(NormActParams p) {
    __shared__ __attribute__((aligned(16))) float lds_mean[kMaxThreads * 8], lds_m2[kMaxThreads * 8];
    const Cut a = p.cut;
    const int chunk = blockIdx.x, slab = blockIdx.y, b = blockIdx.z;
    const int lo = (int)((int64_t)a.N * chunk / a.chunks), hi = (int)((int64_t)a.N * (chunk + 1) / a.chunks);
    const Place at = place_of(a, slab);
    const T* x = (const T*)p.x + (int64_t)b * a.N * a.C + at.c0;
    float mean[8], m2[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) mean[e] = m2[e] = 0.f;
    float n = 0.f;
    if (at.in) {
        Rows<T, ROWS> xs;
        int t = lo + at.r;
        xs.begin(x, t, hi, a);
        for (; t < hi; t += a.RP * ROWS, xs.step()) {
            xs.ahead(x, t, hi, a);
            float v[ROWS][8];
            int rows = 0;
#pragma unroll
            for (int i = 0; i < ROWS; ++i) {
                const bool here = t + i * a.RP < hi;
                xs.cur[i].get(v[i]);
#pragma unroll
                for (int e = 0; e < 8; ++e) v[i][e] = here ? v[i][e] : 0.f;
                rows += here;
            }
            const float cnt = (float)rows, total = n + cnt;
            const float share = cnt / total, both = n * share;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                float s = 0.f, q = 0.f;
#pragma unroll
                for (int i = 0; i < ROWS; ++i) s += v[i][e];
                const float m = s / cnt;
#pragma unroll
                for (int i = 0; i < ROWS; ++i) {
                    const float d = i < rows ? v[i][e] - m : 0.f;
                    q = __builtin_fmaf(d, d, q);
                }
                const float d = m - mean[e];
                mean[e] = __builtin_fmaf(d, share, mean[e]);
                m2[e] += __builtin_fmaf(d * d, both, q);
            }
            n = total;
        }
        store8(lds_mean + at.r * a.S + 8 * at.v, mean);
        store8(lds_m2 + at.r * a.S + 8 * at.v, m2);
    }
    __syncthreads();
    // A group's entries: RP row lanes of its channels.
    const int T_ = group_lanes(a.threads, a.gs);
    const int g = threadIdx.x / T_, l = threadIdx.x % T_;
    const bool mine = g < a.gs;
    const int entries = mine ? a.RP * a.cg : 0;
    const float inv_cg = 1.f / (float)a.cg;
    auto rows_of = [&](int r) { return (float)max(0, (hi - lo - r + a.RP - 1) / a.RP); };
    float sum = 0.f;
    for (int i = l; i < entries; i += T_) {
        const int r = group_of(i, inv_cg), c = g * a.cg + i - r * a.cg;
        sum = __builtin_fmaf(rows_of(r), lds_mean[r * a.S + c], sum);
    }
    const float count = (float)(hi - lo) * (float)a.cg;
    const float gm = lanes_sum(sum, T_) / count;
    float q = 0.f;
    for (int i = l; i < entries; i += T_) {
        const int r = group_of(i, inv_cg), c = g * a.cg + i - r * a.cg;
        const float d = lds_mean[r * a.S + c] - gm;
        q += __builtin_fmaf(d * d, rows_of(r), lds_m2[r * a.S + c]);
    }
    q = lanes_sum(q, T_);
    if (mine && l == 0) {
        float* o = p.records + (((int64_t)b * a.chunks + chunk) * a.G + slab * a.gs + g) * 3;
        o[0] = count;
        o[1] = gm;
        o[2] = q;
    }
}

// The records of more than kFewChunks chunks as one: a workgroup to a group, and
// a thread to two records, so that all are on their way at once.
constexpr int kMergeThreads = 256;
static_assert(kBlocks <= 2 * kMergeThreads, "two records a thread");

// The sum of v over the workgroup.
__device__ __forceinline__ float block_sum(float v, float* lds) {
    v = lanes_sum(v, 64);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
    __syncthreads();
    float t = 0.f;
#pragma unroll
    for (int w = 0; w < kMergeThreads / 64; ++w) t += lds[w];
    return t;
}
__global__ __launch_bounds__(kMergeThreads) void norm_act_merge_stats(NormActParams p) {
    __shared__ float lds[kMergeThreads / 64];
    const Cut a = p.cut;
    const int g = blockIdx.x, b = blockIdx.y;
    const float* rec = p.records + ((int64_t)b * a.chunks * a.G + g) * 3;
    const float count = (float)a.N * (float)a.cg;
    float r[2][3];
#pragma unroll
    for (int u = 0; u < 2; ++u) {
        const int i = threadIdx.x + u * kMergeThreads;
#pragma unroll
        for (int k = 0; k < 3; ++k) r[u][k] = i < a.chunks ? rec[(int64_t)i * a.G * 3 + k] : 0.f;
    }
    const float m = block_sum(__builtin_fmaf(r[0][0], r[0][1], r[1][0] * r[1][1]), lds) / count;
    float q = 0.f;
#pragma unroll
    for (int u = 0; u < 2; ++u) {
        const float d = r[u][1] - m;
        q += __builtin_fmaf(d * d, r[u][0], r[u][2]);
    }
    q = block_sum(q, lds);
    if (threadIdx.x == 0) {
        float* o = p.merged + ((int64_t)b * a.G + g) * 3;
        o[0] = count;
        o[1] = m;
        o[2] = q;
    }
}
__global__ __launch_bounds__(kMergeThreads) void norm_act_merge_sums(NormActParams p) {
    __shared__ float lds[kMergeThreads / 64];
    const Cut a = p.cut;
    const int g = blockIdx.x, b = blockIdx.y;
    const float* rec = p.records + ((int64_t)b * a.chunks * a.G + g) * 2;
    float s[2] = {0.f, 0.f};
#pragma unroll
    for (int u = 0; u < 2; ++u) {
        const int i = threadIdx.x + u * kMergeThreads;
#pragma unroll
        for (int k = 0; k < 2; ++k) s[k] += i < a.chunks ? rec[(int64_t)i * a.G * 2 + k] : 0.f;
    }
    s[0] = block_sum(s[0], lds);
    s[1] = block_sum(s[1], lds);
    if (threadIdx.x == 0) {
        float* o = p.merged + ((int64_t)b * a.G + g) * 2;
        o[0] = s[0];
        o[1] = s[1];
    }
}

// ---- forward ----

template <int ACT>
__device__ __forceinline__ float act_of(float z, float* grad) {
    if constexpr (ACT == PCPP_ACT_NONE) {
        if (grad) *grad = 1.f;
        return z;
    } else {
        return ff_act<ACT>(z, grad);
    }
}

template <typename T, int ACT, int ROWS>
__global__ __launch_bounds__(kMaxThreads) void norm_act_apply(NormActParams p) {
    __shared__ float g_mean[kMaxGroups], g_rstd[kMaxGroups];
    const Cut a = p.cut;
    const int slab = blockIdx.y, b = blockIdx.z;
    const Place at = place_of(a, slab);
    const int lo = (int)((int64_t)a.N * blockIdx.x / p.apply_blocks), hi = (int)((int64_t)a.N * (blockIdx.x + 1) / p.apply_blocks);
    const int64_t base = (int64_t)b * a.N * a.C + at.c0;
    const T* x = (const T*)p.x + base;
    Rows<T, ROWS> xs;
    int t = lo + at.r;
    if (at.in) xs.begin(x, t, hi, a);  // (on their way while the records are merged)
    {
        const int T_ = group_lanes(a.threads, a.gs);
        const int g = threadIdx.x / T_, l = threadIdx.x % T_;
        const bool mine = g < a.gs;
        const int chunks = p.merged ? 1 : a.chunks;
        const float* rec = (p.merged ? p.merged : p.records) + ((int64_t)b * chunks * a.G + slab * a.gs + (mine ? g : 0)) * 3;
        float sum = 0.f, q = 0.f;
        const float count = (float)a.N * (float)a.cg;
        for (int i = l; i < chunks; i += T_) sum = __builtin_fmaf(rec[(int64_t)i * a.G * 3], rec[(int64_t)i * a.G * 3 + 1], sum);
        const float m = lanes_sum(sum, T_) / count;
        for (int i = l; i < chunks; i += T_) {
            const float* o = rec + (int64_t)i * a.G * 3;
            const float d = o[1] - m;
            q += __builtin_fmaf(d * d, o[0], o[2]);
        }
        q = lanes_sum(q, T_);
        if (mine && l == 0) {
            const float rstd = 1.f / sqrtf(q / count + p.eps);
            g_mean[g] = m;
            g_rstd[g] = rstd;
            if (p.stats != nullptr && blockIdx.x == 0) {
                float* o = p.stats + ((int64_t)b * a.G + slab * a.gs + g) * 2;
                o[0] = m;
                o[1] = rstd;
            }
        }
    }
    __syncthreads();
    if (!at.in) return;
    float mean[8], rstd[8];
    const float inv_cg = 1.f / (float)a.cg;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const int g = group_of(8 * at.v + e, inv_cg);
        mean[e] = g_mean[g];
        rstd[e] = g_rstd[g];
    }
    const bf16x8 gamma = *(const bf16x8*)(p.gamma + at.c0), beta = *(const bf16x8*)(p.beta + at.c0);
    const DropoutKey key = dropout_key(p.drop);
    for (; t < hi; t += a.RP * ROWS, xs.step()) {
        xs.ahead(x, t, hi, a);
#pragma unroll
        for (int i = 0; i < ROWS; ++i) {
            if (t + i * a.RP >= hi) break;
            const int64_t o = base + (int64_t)(t + i * a.RP) * a.C;
            float v[8];
            xs.cur[i].get(v);
#pragma unroll
            for (int e = 0; e < 8; ++e)
                v[e] = act_of<ACT>(__builtin_fmaf((v[e] - mean[e]) * rstd[e], bf16_to_f32(gamma[e]), bf16_to_f32(beta[e])), nullptr);
            if (p.drop.least > 0) drop8(p.drop, key, (uint64_t)o / 8, v);
            store8((T*)p.y + o, v);
        }
    }
}

// ---- backward ----

// A thread's channels.
struct Channels {
    float mean[8], rstd[8];
    bf16x8 gamma, beta;
    __device__ __forceinline__ Channels(const NormActParams& p, const Place& at, int slab, int b) {
        const Cut& a = p.cut;
        const float inv_cg = 1.f / (float)a.cg;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float* s = p.stats + ((int64_t)b * a.G + slab * a.gs + group_of(8 * at.v + e, inv_cg)) * 2;
            mean[e] = s[0];
            rstd[e] = s[1];
        }
        gamma = *(const bf16x8*)(p.gamma + at.c0);
        beta = *(const bf16x8*)(p.beta + at.c0);
    }
};

// Eight channels of the row at o: v, x, becomes n; d, dy, becomes g but for
// dropout's factor, which all have in common.
template <int ACT>
__device__ __forceinline__ void grad8(const NormActParams& p, const DropoutKey& key, int64_t o, const Channels& c,
                                      float (&v)[8], float (&d)[8]) {
    if (p.drop.least > 0) keep8(p.drop, key, (uint64_t)o / 8, d);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        v[e] = (v[e] - c.mean[e]) * c.rstd[e];
        float da;
        act_of<ACT>(__builtin_fmaf(v[e], bf16_to_f32(c.gamma[e]), bf16_to_f32(c.beta[e])), &da);
        d[e] *= da;
    }
}

template <typename T, int ACT, int ROWS>
__global__ __launch_bounds__(kMaxThreads) void norm_act_grad_sums(NormActParams p) {
    __shared__ __attribute__((aligned(16))) float lds_n[kMaxThreads * 8], lds_g[kMaxThreads * 8];
    const Cut a = p.cut;
    const int chunk = blockIdx.x, slab = blockIdx.y, b = blockIdx.z;
    const int lo = (int)((int64_t)a.N * chunk / a.chunks), hi = (int)((int64_t)a.N * (chunk + 1) / a.chunks);
    const Place at = place_of(a, slab);
    if (at.in) {
        const int64_t base = (int64_t)b * a.N * a.C + at.c0;
        const T *x = (const T*)p.x + base, *dy = (const T*)p.dy + base;
        Rows<T, ROWS> xs, ds;
        int t = lo + at.r;
        xs.begin(x, t, hi, a);
        ds.begin(dy, t, hi, a);
        const Channels ch(p, at, slab, b);
        float sn[8], sg[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) sn[e] = sg[e] = 0.f;
        const DropoutKey key = dropout_key(p.drop);
        for (; t < hi; t += a.RP * ROWS, xs.step(), ds.step()) {
            xs.ahead(x, t, hi, a);
            ds.ahead(dy, t, hi, a);
#pragma unroll
            for (int i = 0; i < ROWS; ++i) {
                if (t + i * a.RP >= hi) break;
                float v[8], d[8];
                xs.cur[i].get(v);
                ds.cur[i].get(d);
                grad8<ACT>(p, key, base + (int64_t)(t + i * a.RP) * a.C, ch, v, d);
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    sn[e] = __builtin_fmaf(d[e], v[e], sn[e]);
                    sg[e] += d[e];
                }
            }
        }
        store8(lds_n + at.r * a.S + 8 * at.v, sn);
        store8(lds_g + at.r * a.S + 8 * at.v, sg);
    }
    __syncthreads();
    for (int c = threadIdx.x; c < a.S; c += a.threads) {
        float tn = 0.f, tg = 0.f;
        for (int r = 0; r < a.RP; ++r) {
            tn += lds_n[r * a.S + c];
            tg += lds_g[r * a.S + c];
        }
        if (p.drop.least > 0) {
            tn *= p.drop.factor;
            tg *= p.drop.factor;
        }
        if (p.columns != nullptr) {
            float* o = p.columns + ((int64_t)b * a.chunks + chunk) * a.C + slab * a.S + c;
            o[0] = tn;
            o[(int64_t)a.B * a.chunks * a.C] = tg;
        }
        const float gamma = bf16_to_f32(p.gamma[slab * a.S + c]);
        lds_n[c] = tn * gamma;  // row 0, which this thread alone has read
        lds_g[c] = tg * gamma;
    }
    __syncthreads();
    const int T_ = group_lanes(a.threads, a.gs);
    const int g = threadIdx.x / T_, l = threadIdx.x % T_;
    const bool mine = g < a.gs;
    float s0 = 0.f, s1 = 0.f;
    if (mine)
        for (int c = l; c < a.cg; c += T_) {
            s0 += lds_g[g * a.cg + c];
            s1 += lds_n[g * a.cg + c];
        }
    s0 = lanes_sum(s0, T_);
    s1 = lanes_sum(s1, T_);
    if (mine && l == 0) {
        float* o = p.records + (((int64_t)b * a.chunks + chunk) * a.G + slab * a.gs + g) * 2;
        o[0] = s0;
        o[1] = s1;
    }
}

// dgamma and dbeta of 16 channels: the chunks' sums in a fixed order.
__device__ __forceinline__ void column_totals(const NormActParams& p, int block, float* lds) {
    const Cut& a = p.cut;
    const int per = (a.C + 15) / 16, which = block / per;
    const int l = threadIdx.x & 15, r = threadIdx.x >> 4, lanes = a.threads >> 4;
    const int c = 16 * (block - which * per) + l, rows = a.B * a.chunks;
    const float* in = p.columns + (int64_t)which * rows * a.C;
    float t = 0.f;
    if (c < a.C) {
        int i = r;
        for (; i + 7 * lanes < rows; i += 8 * lanes) {
            float v[8];
#pragma unroll
            for (int u = 0; u < 8; ++u) v[u] = in[(int64_t)(i + u * lanes) * a.C + c];
#pragma unroll
            for (int u = 0; u < 8; ++u) t += v[u];
        }
        for (; i < rows; i += lanes) t += in[(int64_t)i * a.C + c];
    }
    lds[17 * r + l] = t;
    __syncthreads();
    bf16* out = which ? p.dbeta : p.dgamma;
    if (r == 0 && c < a.C && out != nullptr) {
        float v = 0.f;
        for (int i = 0; i < lanes; ++i) v += lds[17 * i + l];
        out[c] = f32_to_bf16(v);
    }
}
int column_blocks(const NormActParams& p) { return p.columns != nullptr ? 2 * ((p.cut.C + 15) / 16) : 0; }

// blockIdx.x: apply_blocks x slabs x images, then the columns' totals.
template <typename T, int ACT, int ROWS>
__global__ __launch_bounds__(kMaxThreads) void norm_act_grad_apply(NormActParams p) {
    __shared__ float lds[17 * (kMaxThreads / 16)];
    __shared__ float g_m0[kMaxGroups], g_m1[kMaxGroups];
    const Cut a = p.cut;
    const int slabs = a.C / a.S;
    const int64_t applying = (int64_t)p.apply_blocks * slabs * a.B;
    if (blockIdx.x >= applying) {
        column_totals(p, (int)(blockIdx.x - applying), lds);
        return;
    }
    const int part = (int)(blockIdx.x % p.apply_blocks), sb = (int)(blockIdx.x / p.apply_blocks);
    const int slab = sb % slabs, b = sb / slabs;
    const Place at = place_of(a, slab);
    const int lo = (int)((int64_t)a.N * part / p.apply_blocks), hi = (int)((int64_t)a.N * (part + 1) / p.apply_blocks);
    const int64_t base = (int64_t)b * a.N * a.C + at.c0;
    const T *x = (const T*)p.x + base, *dy = (const T*)p.dy + base;
    Rows<T, ROWS> xs, ds;
    int t = lo + at.r;
    if (at.in) {  // (on their way while the records are merged)
        xs.begin(x, t, hi, a);
        ds.begin(dy, t, hi, a);
    }
    {
        const int T_ = group_lanes(a.threads, a.gs);
        const int g = threadIdx.x / T_, l = threadIdx.x % T_;
        const bool mine = g < a.gs;
        const int chunks = p.merged ? 1 : a.chunks;
        const float* rec = (p.merged ? p.merged : p.records) + ((int64_t)b * chunks * a.G + slab * a.gs + (mine ? g : 0)) * 2;
        float s0 = 0.f, s1 = 0.f;
        for (int i = l; i < chunks; i += T_) {
            s0 += rec[(int64_t)i * a.G * 2];
            s1 += rec[(int64_t)i * a.G * 2 + 1];
        }
        s0 = lanes_sum(s0, T_);
        s1 = lanes_sum(s1, T_);
        if (mine && l == 0) {
            const float count = (float)a.N * (float)a.cg;
            g_m0[g] = s0 / count;
            g_m1[g] = s1 / count;
        }
    }
    __syncthreads();
    if (!at.in) return;
    const Channels ch(p, at, slab, b);
    float m0[8], m1[8], gamma[8];
    const float inv_cg = 1.f / (float)a.cg;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const int g = group_of(8 * at.v + e, inv_cg);
        m0[e] = g_m0[g];
        m1[e] = g_m1[g];
        gamma[e] = bf16_to_f32(ch.gamma[e]) * (p.drop.least > 0 ? p.drop.factor : 1.f);
    }
    const DropoutKey key = dropout_key(p.drop);
    for (; t < hi; t += a.RP * ROWS, xs.step(), ds.step()) {
        xs.ahead(x, t, hi, a);
        ds.ahead(dy, t, hi, a);
#pragma unroll
        for (int i = 0; i < ROWS; ++i) {
            if (t + i * a.RP >= hi) break;
            const int64_t o = base + (int64_t)(t + i * a.RP) * a.C;
            float v[8], d[8];
            xs.cur[i].get(v);
            ds.cur[i].get(d);
            grad8<ACT>(p, key, o, ch, v, d);
#pragma unroll
            for (int e = 0; e < 8; ++e) d[e] = ch.rstd[e] * (__builtin_fmaf(d[e], gamma[e], -m0[e]) - v[e] * m1[e]);
            store8((T*)p.y + o, d);
        }
    }
}

// ---- few tokens: a slab of an image in one workgroup's registers, one launch ----

// The sum of v over the wavefronts of the thread's group: as many to each
// of the slab's gs groups (1, 2, 4 or 8 of them).
__device__ __forceinline__ float group_total(const Cut& a, float v, float* lds) {
    const int waves = a.threads / 64 / a.gs, wave = threadIdx.x >> 6;
    v = lanes_sum(v, 64);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) lds[wave] = v;
    __syncthreads();
    float t = 0.f;
    for (int w = 0; w < waves; ++w) t += lds[wave / waves * waves + w];
    return t;
}
// Per-channel values of all threads, in part [RP][S], summed over the rows and
// channels of the thread's group of wavefronts.
__device__ __forceinline__ float group_share(const Cut& a, const float (&v)[8], const Place& at, float* part) {
    if (a.gs == 1) {
        float t = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) t += v[e];
        return t;  // (0 of the threads left over)
    }
    __syncthreads();
    if (at.in) store8(part + at.r * a.S + 8 * at.v, v);
    __syncthreads();
    const int lanes = a.threads / a.gs, g = threadIdx.x / lanes;
    const float inv_cg = 1.f / (float)a.cg;
    float t = 0.f;
    for (int i = threadIdx.x % lanes; i < a.RP * a.cg; i += lanes) {
        const int r = group_of(i, inv_cg);
        t += part[r * a.S + g * a.cg + i - r * a.cg];
    }
    return t;
}

// Mean by the sum, then the deviations from it: their squares, and their sum for
// what the mean is off by.
template <typename T, int ACT>
__global__ __launch_bounds__(kMaxThreads) void norm_act_whole(NormActParams p) {
    __shared__ __attribute__((aligned(16))) float part[kMaxThreads * 8];
    __shared__ float lds[kMaxThreads / 64], g_mean[8], g_rstd[8];
    const Cut a = p.cut;
    const int slab = blockIdx.x, b = blockIdx.y;
    const Place at = place_of(a, slab);
    const int64_t base = (int64_t)b * a.N * a.C + at.c0;
    Raw<T> x[kWholeRows];
    float s[8], q[8], mean[8], rstd[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) s[e] = q[e] = 0.f;
    if (at.in) {
#pragma unroll
        for (int i = 0; i < kWholeRows; ++i)
            if (at.r + i * a.RP < a.N) x[i].load((const T*)p.x + base + (int64_t)(at.r + i * a.RP) * a.C);
#pragma unroll
        for (int i = 0; i < kWholeRows; ++i)
            if (at.r + i * a.RP < a.N) {
                float v[8];
                x[i].get(v);
#pragma unroll
                for (int e = 0; e < 8; ++e) s[e] += v[e];
            }
    }
    const float count = (float)a.N * (float)a.cg, inv_cg = 1.f / (float)a.cg;
    const int lanes = kMaxThreads / a.gs, g = threadIdx.x / lanes;
    const bool first = threadIdx.x % lanes == 0;
    const float m = group_total(a, group_share(a, s, at, part), lds) / count;
    if (first) g_mean[g] = m;
    __syncthreads();
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        mean[e] = at.in ? g_mean[group_of(8 * at.v + e, inv_cg)] : 0.f;
        s[e] = 0.f;
    }
    if (at.in) {
#pragma unroll
        for (int i = 0; i < kWholeRows; ++i)
            if (at.r + i * a.RP < a.N) {
                float v[8];
                x[i].get(v);
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const float d = v[e] - mean[e];
                    s[e] += d;
                    q[e] = __builtin_fmaf(d, d, q[e]);
                }
            }
    }
    const float off = group_total(a, group_share(a, s, at, part), lds) / count;
    const float var = group_total(a, group_share(a, q, at, part), lds) / count - off * off;
    if (first) {
        g_mean[g] = m + off;
        g_rstd[g] = 1.f / sqrtf(fmaxf(var, 0.f) + p.eps);
        if (p.stats != nullptr) {
            float* o = p.stats + ((int64_t)b * a.G + slab * a.gs + g) * 2;
            o[0] = g_mean[g];
            o[1] = g_rstd[g];
        }
    }
    __syncthreads();
    if (!at.in) return;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        mean[e] = g_mean[group_of(8 * at.v + e, inv_cg)];
        rstd[e] = g_rstd[group_of(8 * at.v + e, inv_cg)];
    }
    const bf16x8 gamma = *(const bf16x8*)(p.gamma + at.c0), beta = *(const bf16x8*)(p.beta + at.c0);
    const DropoutKey key = dropout_key(p.drop);
#pragma unroll
    for (int i = 0; i < kWholeRows; ++i) {
        if (at.r + i * a.RP >= a.N) break;
        const int64_t o = base + (int64_t)(at.r + i * a.RP) * a.C;
        float v[8];
        x[i].get(v);
#pragma unroll
        for (int e = 0; e < 8; ++e)
            v[e] = act_of<ACT>(__builtin_fmaf((v[e] - mean[e]) * rstd[e], bf16_to_f32(gamma[e]), bf16_to_f32(beta[e])), nullptr);
        if (p.drop.least > 0) drop8(p.drop, key, (uint64_t)o / 8, v);
        store8((T*)p.y + o, v);
    }
}

// The sums of w and w n, and the images' sums of the columns (of the only image:
// dgamma and dbeta themselves).
template <typename T, int ACT>
__global__ __launch_bounds__(kMaxThreads) void norm_act_grad_whole(NormActParams p) {
    __shared__ __attribute__((aligned(16))) float part[2][kMaxThreads * 8];
    __shared__ float lds[kMaxThreads / 64], g_m0[8], g_m1[8];
    const Cut a = p.cut;
    const int slab = blockIdx.x, b = blockIdx.y;
    const Place at = place_of(a, slab);
    const int64_t base = (int64_t)b * a.N * a.C + at.c0;
    Raw<T> x[kGradRows];
    float gr[kGradRows][8];  // dy, then g but for dropout's factor
    const DropoutKey key = dropout_key(p.drop);
    const float factor = p.drop.least > 0 ? p.drop.factor : 1.f;
    const float inv_cg = 1.f / (float)a.cg;
    if (at.in) {
#pragma unroll
        for (int i = 0; i < kGradRows; ++i)
            if (at.r + i * a.RP < a.N) {
                x[i].load((const T*)p.x + base + (int64_t)(at.r + i * a.RP) * a.C);
                load8((const T*)p.dy + base + (int64_t)(at.r + i * a.RP) * a.C, gr[i]);
            }
    }
    const Place safe = at.in ? at : Place{0, 0, slab * a.S, false};
    const Channels ch(p, safe, slab, b);
    float sn[8], sg[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) sn[e] = sg[e] = 0.f;
    if (at.in) {
#pragma unroll
        for (int i = 0; i < kGradRows; ++i)
            if (at.r + i * a.RP < a.N) {
                float v[8];
                x[i].get(v);
                grad8<ACT>(p, key, base + (int64_t)(at.r + i * a.RP) * a.C, ch, v, gr[i]);
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    sn[e] = __builtin_fmaf(gr[i][e], v[e], sn[e]);
                    sg[e] += gr[i][e];
                }
            }
    }
    if (p.dgamma != nullptr || p.dbeta != nullptr) {
        if (at.in) {
            store8(part[0] + at.r * a.S + 8 * at.v, sn);
            store8(part[1] + at.r * a.S + 8 * at.v, sg);
        }
        __syncthreads();
        // every channel by several threads, then their sums
        const int k = group_of(threadIdx.x, 1.f / (float)a.S), c = threadIdx.x - k * a.S, rows = kMaxThreads / a.S;
        float tn = 0.f, tg = 0.f;
        if (k < rows)
            for (int r = k; r < a.RP; r += rows) {
                tn += part[0][r * a.S + c];
                tg += part[1][r * a.S + c];
            }
        __syncthreads();
        if (k < rows) {
            part[0][threadIdx.x] = tn;
            part[1][threadIdx.x] = tg;
        }
        __syncthreads();
        if (threadIdx.x < a.S) {
            for (int r = 1; r < rows; ++r) {
                tn += part[0][r * a.S + c];
                tg += part[1][r * a.S + c];
            }
            tn *= factor;
            tg *= factor;
            const int channel = slab * a.S + c;
            if (p.columns != nullptr) {
                p.columns[(int64_t)b * a.C + channel] = tn;
                p.columns[((int64_t)a.B + b) * a.C + channel] = tg;
            } else {
                if (p.dgamma != nullptr) p.dgamma[channel] = f32_to_bf16(tn);
                if (p.dbeta != nullptr) p.dbeta[channel] = f32_to_bf16(tg);
            }
        }
    }
    float gamma[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        gamma[e] = bf16_to_f32(ch.gamma[e]) * factor;
        sn[e] *= gamma[e];
        sg[e] *= gamma[e];
    }
    const float count = (float)a.N * (float)a.cg;
    const float t0 = group_total(a, group_share(a, sg, at, part[0]), lds) / count;
    const float t1 = group_total(a, group_share(a, sn, at, part[0]), lds) / count;
    const int lanes = kMaxThreads / a.gs;
    if (threadIdx.x % lanes == 0) {
        g_m0[threadIdx.x / lanes] = t0;
        g_m1[threadIdx.x / lanes] = t1;
    }
    __syncthreads();
    if (!at.in) return;
    float m0[8], m1[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        m0[e] = g_m0[group_of(8 * at.v + e, inv_cg)];
        m1[e] = g_m1[group_of(8 * at.v + e, inv_cg)];
    }
#pragma unroll
    for (int i = 0; i < kGradRows; ++i) {
        if (at.r + i * a.RP >= a.N) break;
        const int64_t o = base + (int64_t)(at.r + i * a.RP) * a.C;
        float v[8];
        x[i].get(v);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float n = (v[e] - ch.mean[e]) * ch.rstd[e];
            v[e] = ch.rstd[e] * (__builtin_fmaf(gr[i][e], gamma[e], -m0[e]) - n * m1[e]);
        }
        store8((T*)p.y + o, v);
    }
}

__global__ __launch_bounds__(kMaxThreads) void norm_act_columns(NormActParams p) {
    __shared__ float lds[17 * (kMaxThreads / 16)];
    column_totals(p, (int)blockIdx.x, lds);
}

int gcd_of(int a, int b) { return b == 0 ? a : gcd_of(b, a % b); }

// Whole rows where the tokens alone make enough workgroups: every row is one run
// of memory.  Else slabs, as wide as still give the chip its workgroups.  256
// threads, though some of them may be idle (2 x 57600 x 640 bf16 with 240 of 256
// at work 288 us forward and backward, with 320 of 320 at work 348).
Cut cut_of(int B, int N, int C, int G) {
    Cut best = {};
    const int cg = C / G, least = 8 / gcd_of(8, cg);  // groups whose channels are whole vectors; divides G as 8 divides C
    for (int gs = G; gs >= least; --gs) {
        if (G % gs != 0 || gs % least != 0) continue;
        Cut a = {B, N, C, G, cg, gs * cg, gs * cg / 8, 0, gs, 0, 256};
        if (a.V > 256) a.threads = kMaxThreads;
        a.RP = a.threads / a.V;
        const int64_t fit = (N + kRunRows * a.RP - 1) / (kRunRows * a.RP);
        if (gs == G && B * fit >= kBlocks) {
            const int64_t most = (kBlocks + B - 1) / B;
            a.chunks = (int)(fit < most ? fit : most);
            return a;
        }
        a.chunks = (int)(fit < kFewChunks ? fit : kFewChunks);
        if (best.B != 0 && (a.V < 8 || 5 * a.V * a.RP < 4 * best.V * best.RP)) continue;
        best = a;
        if ((int64_t)B * (G / gs) * a.chunks >= kBlocks) break;
    }
    return best;
}

// The least slab, if a workgroup's registers hold it of all tokens and there are
// not more workgroups than compute units; else V = 0.  A workgroup of such a
// slab then does on its own, in one launch, what else the whole chip does in
// two: faster as long as that is little.  2 x 64 x 1280 bf16 5.7 us forward and
// 8.4 backward (else 12.9 and 12.0), 2 x 512 x 1280 9.6 and 13.4 (13.9 and
// 14.9), 8 x 512 x 1280 14.0 and 21.6 (19.5 and 31.0); with the groups of 10
// channels of 1 x 800 x 320, eight rows of four groups, 13.3 and 15.1 (11.3 and
// 14.4); with 2048 workgroups, 64 x 256 x 1280, 40 and 87 (40 and 62).
Cut whole_of(int B, int N, int C, int G, int rows) {
    const int cg = C / G, gs = 8 / gcd_of(8, cg);
    Cut a = {B, N, C, G, cg, gs * cg, gs * cg / 8, 0, gs, 1, kMaxThreads};
    a.RP = a.threads / a.V;
    if (a.V < kWholeVectors || a.S > kMaxThreads || N > (gs == 1 ? rows : rows / 2) * a.RP || (int64_t)B * (C / a.S) > kWholeBlocks) a.V = 0;
    return a;
}

// Rows of a thread of the apply launches: enough workgroups first.
int apply_blocks_of(const Cut& a) {
    const int64_t most = (a.N + 4 * a.RP - 1) / (4 * a.RP), slabs = (int64_t)a.B * (a.C / a.S);
    int64_t n = (2048 + slabs - 1) / slabs;
    n = n < most ? n : most;
    return (int)(n > 0 ? n : 1);
}

// [merged][records], and backward [columns].
int64_t merged_floats(const Cut& a) { return ((int64_t)a.B * a.G * 3 + 3) / 4 * 4; }
int64_t stats_floats(const Cut& a) { return merged_floats(a) + (int64_t)a.B * a.chunks * a.G * 3; }
int64_t grad_records(const Cut& a) { return (int64_t)a.B * a.chunks * 2 * a.G; }
int64_t grad_floats(const Cut& a) { return merged_floats(a) + grad_records(a) + (int64_t)a.B * a.chunks * 2 * a.C; }

template <typename F>
void with_act(int act, F f) {
    using std::integral_constant;
    if (act == PCPP_ACT_SILU) f(integral_constant<int, PCPP_ACT_SILU>());
    else if (act == PCPP_ACT_GELU) f(integral_constant<int, PCPP_ACT_GELU>());
    else f(integral_constant<int, PCPP_ACT_NONE>());
}

int check_geom(const pcpp_norm_act_geom_t* g) {
    if (!g || g->reserved != 0) return PCPP_EINVAL;
    if (g->batch < 1 || g->batch > 65535 || g->tokens < 1 || g->tokens > kMaxTokens || g->channels < 1 || g->groups < 1) return PCPP_EINVAL;
    if (!(g->eps > 0.f) || !(g->drop >= 0.f && g->drop <= 1.f)) return PCPP_EINVAL;
    if (g->dtype != PCPP_DTYPE_F32 && g->dtype != PCPP_DTYPE_BF16) return PCPP_ENOTSUP;
    if (g->act != PCPP_ACT_GELU && g->act != PCPP_ACT_SILU && g->act != PCPP_ACT_NONE) return PCPP_ENOTSUP;
    if (!gn_shapes_ok(g->channels, g->groups)) return PCPP_ENOTSUP;
    if ((int64_t)g->batch * g->tokens > ((int64_t)1 << 36) / g->channels) return PCPP_EINVAL;
    return PCPP_OK;
}

}  // namespace

}  // namespace pcpp

using namespace pcpp;

PCPP_EXPORT size_t pcpp_group_norm_act_workspace_size(const pcpp_norm_act_geom_t* g) {
    if (check_geom(g) != PCPP_OK) return 0;
    const Cut a = cut_of(g->batch, g->tokens, g->channels, g->groups);
    const int64_t f = stats_floats(a), b = grad_floats(a);
    return (size_t)(f > b ? f : b) * sizeof(float);
}

PCPP_EXPORT int pcpp_group_norm_act(const pcpp_norm_act_geom_t* g, const void* x, const void* gamma, const void* beta,
                                    const void* rng, uint64_t draw, void* y, float* stats, void* workspace,
                                    size_t ws_bytes, void* stream) {
    const int st = check_geom(g);
    if (st != PCPP_OK) return st;
    if (!x || !gamma || !beta || !y || (g->drop > 0.f && !rng)) return PCPP_EINVAL;
    const void* ptrs[] = {x, gamma, beta, y};
    for (const void* q : ptrs)
        if (!aligned_to(q, 16)) return PCPP_EINVAL;
    if (!aligned_to(stats, 4) || !aligned_to(rng, 8)) return PCPP_EINVAL;
    if (!workspace || ws_bytes < pcpp_group_norm_act_workspace_size(g)) return PCPP_EWORKSPACE;
    if (!aligned_to(workspace, 16)) return PCPP_EINVAL;
    const int64_t n = (int64_t)g->batch * g->tokens * g->channels, size = g->dtype == PCPP_DTYPE_F32 ? 4 : 2;
    const int64_t cb = 2 * (int64_t)g->channels, sb = 8 * (int64_t)g->batch * g->groups;
    const Range out[] = {{y, n * size}, {stats, sb}, {workspace, (int64_t)pcpp_group_norm_act_workspace_size(g)}};
    const Range in[] = {{x, n * size}, {gamma, cb}, {beta, cb}, {rng, 16}};
    if (outputs_overlap(out, 3, in, 4)) return PCPP_EINVAL;
    const Cut a = cut_of(g->batch, g->tokens, g->channels, g->groups);
    NormActParams p = {};
    p.x = x;
    p.gamma = (const bf16*)gamma;
    p.beta = (const bf16*)beta;
    p.y = y;
    p.stats = stats;
    p.records = (float*)workspace + merged_floats(a);
    p.merged = a.chunks > kFewChunks ? (float*)workspace : nullptr;
    p.drop = make_dropout(g->drop, rng, draw);
    p.cut = a;
    p.apply_blocks = apply_blocks_of(a);
    p.eps = g->eps;
    const hipStream_t s = (hipStream_t)stream;
    const Cut whole = whole_of(g->batch, g->tokens, g->channels, g->groups, kWholeRows);
    if (whole.V > 0) {
        p.cut = whole;
        with_act(g->act, [&](auto act) {
            const dim3 grid(whole.C / whole.S, whole.B);
            if (g->dtype == PCPP_DTYPE_F32)
                norm_act_whole<float, act()><<<grid, whole.threads, 0, s>>>(p);
            else
                norm_act_whole<bf16, act()><<<grid, whole.threads, 0, s>>>(p);
        });
        return hipGetLastError() == hipSuccess ? PCPP_OK : PCPP_EHIP;
    }
    const dim3 sums(a.chunks, a.C / a.S, a.B), apply(p.apply_blocks, a.C / a.S, a.B);
    if (g->dtype == PCPP_DTYPE_F32)
        norm_act_stats<float, kRunRows / 2><<<sums, a.threads, 0, s>>>(p);
    else
        norm_act_stats<bf16, kRunRows><<<sums, a.threads, 0, s>>>(p);
    if (p.merged) norm_act_merge_stats<<<dim3(a.G, a.B), kMergeThreads, 0, s>>>(p);
    if (hipGetLastError() != hipSuccess) return PCPP_EHIP;
    with_act(g->act, [&](auto act) {
        if (g->dtype == PCPP_DTYPE_F32)
            norm_act_apply<float, act(), 2><<<apply, a.threads, 0, s>>>(p);
        else
            norm_act_apply<bf16, act(), 4><<<apply, a.threads, 0, s>>>(p);
    });
    return hipGetLastError() == hipSuccess ? PCPP_OK : PCPP_EHIP;
}

PCPP_EXPORT int pcpp_group_norm_act_backward(const pcpp_norm_act_geom_t* g, const void* x, const void* gamma,
                                             const void* beta, const float* stats, const void* rng, uint64_t draw,
                                             const void* dy, void* dx, void* dgamma, void* dbeta, void* workspace,
                                             size_t ws_bytes, void* stream) {
    const int st = check_geom(g);
    if (st != PCPP_OK) return st;
    if (!x || !gamma || !beta || !stats || !dy || !dx || (g->drop > 0.f && !rng)) return PCPP_EINVAL;
    const void* ptrs[] = {x, gamma, beta, dy, dx, dgamma, dbeta};
    for (const void* q : ptrs)
        if (!aligned_to(q, 16)) return PCPP_EINVAL;
    if (!aligned_to(stats, 4) || !aligned_to(rng, 8)) return PCPP_EINVAL;
    if (!workspace || ws_bytes < pcpp_group_norm_act_workspace_size(g)) return PCPP_EWORKSPACE;
    if (!aligned_to(workspace, 16)) return PCPP_EINVAL;
    const int64_t n = (int64_t)g->batch * g->tokens * g->channels, size = g->dtype == PCPP_DTYPE_F32 ? 4 : 2;
    const int64_t cb = 2 * (int64_t)g->channels, sb = 8 * (int64_t)g->batch * g->groups;
    // dx may replace dy: every element is read and written by one lane
    const Range out[] = {{dx, n * size}, {dgamma, cb}, {dbeta, cb}, {workspace, (int64_t)pcpp_group_norm_act_workspace_size(g)}};
    const Range in[] = {{x, n * size}, {gamma, cb}, {beta, cb}, {stats, sb}, {rng, 16}, {dy, n * size}};
    if (outputs_overlap(out, 4, in, dx == dy ? 5 : 6)) return PCPP_EINVAL;
    if (dx == dy && outputs_overlap(out + 1, 3, in + 5, 1)) return PCPP_EINVAL;
    const Cut a = cut_of(g->batch, g->tokens, g->channels, g->groups);
    NormActParams p = {};
    p.x = x;
    p.dy = dy;
    p.gamma = (const bf16*)gamma;
    p.beta = (const bf16*)beta;
    p.y = dx;
    p.stats = (float*)stats;
    p.records = (float*)workspace + merged_floats(a);
    p.merged = a.chunks > kFewChunks ? (float*)workspace : nullptr;
    p.columns = dgamma || dbeta ? p.records + grad_records(a) : nullptr;
    p.dgamma = (bf16*)dgamma;
    p.dbeta = (bf16*)dbeta;
    p.drop = make_dropout(g->drop, rng, draw);
    p.cut = a;
    p.apply_blocks = apply_blocks_of(a);
    const hipStream_t s = (hipStream_t)stream;
    const Cut whole = whole_of(g->batch, g->tokens, g->channels, g->groups, kGradRows);
    if (whole.V > 0) {
        p.cut = whole;
        p.columns = (dgamma || dbeta) && whole.B > 1 ? (float*)workspace : nullptr;
        with_act(g->act, [&](auto act) {
            const dim3 grid(whole.C / whole.S, whole.B);
            if (g->dtype == PCPP_DTYPE_F32)
                norm_act_grad_whole<float, act()><<<grid, whole.threads, 0, s>>>(p);
            else
                norm_act_grad_whole<bf16, act()><<<grid, whole.threads, 0, s>>>(p);
        });
        if (p.columns) norm_act_columns<<<column_blocks(p), whole.threads, 0, s>>>(p);
        return hipGetLastError() == hipSuccess ? PCPP_OK : PCPP_EHIP;
    }
    const dim3 sums(a.chunks, a.C / a.S, a.B);
    const int64_t blocks = (int64_t)p.apply_blocks * (a.C / a.S) * a.B + column_blocks(p);
    with_act(g->act, [&](auto act) {
        if (g->dtype == PCPP_DTYPE_F32)
            norm_act_grad_sums<float, act(), 1><<<sums, a.threads, 0, s>>>(p);
        else
            norm_act_grad_sums<bf16, act(), 2><<<sums, a.threads, 0, s>>>(p);
    });
    if (p.merged) norm_act_merge_sums<<<dim3(a.G, a.B), kMergeThreads, 0, s>>>(p);
    if (hipGetLastError() != hipSuccess) return PCPP_EHIP;
    with_act(g->act, [&](auto act) {
        if (g->dtype == PCPP_DTYPE_F32)
            norm_act_grad_apply<float, act(), 1><<<(unsigned)blocks, a.threads, 0, s>>>(p);
        else
            norm_act_grad_apply<bf16, act(), 2><<<(unsigned)blocks, a.threads, 0, s>>>(p);
    });
    return hipGetLastError() == hipSuccess ? PCPP_OK : PCPP_EHIP;
}

// What the masked attention's kernels share: a call's parameters, the mask,
// the scores' transform and the operands of the matrix products.
//
// A product takes 32 x 32 tiles with the queries or the keys of a wavefront in
// the lanes: of the scores' tile a lane holds one column (lane % 32) and the
// rows 8 (r / 4) + 4 (lane / 32) + r % 4 in register r.  Those registers, eight
// at a time and rounded to bf16, are the second operand of the next product as
// they stand, if its first operand takes the contracted rows in the same order:
// row_operand and column_operand do.
#pragma once

#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include "common.h"

namespace pcpp {
namespace masked {

constexpr int TILE = 64;             // tokens of a tile of keys or queries
constexpr float LOG2E = 1.4426950408889634f;
constexpr float LN2 = 0.69314718055994531f;

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

// Documents of 64 tokens: the least and the largest number (lo < 0: some are
// none; hi < 0: all are).
struct DocRange {
    int32_t lo, hi;
};

struct Params {
    const bf16 *q, *k, *v, *dy;
    bf16* y;
    float* lse;                    // [B, H, nq] natural logarithms, or null
    bf16 *dq, *dk, *dv;
    float* delta;                  // [B, H, nq] dy . y
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
    // few queries: pieces of the keys, their results
    int32_t pieces, row_blocks;
    float* part_o;
    float* part_ml;
};

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

__device__ __forceinline__ bool ranges_meet(const DocRange& a, const DocRange& b) {
    return a.hi >= max(b.lo, 0) && b.hi >= max(a.lo, 0);
}
__device__ __forceinline__ bool same_document(const DocRange& a, const DocRange& b) {
    return a.lo >= 0 && a.lo == a.hi && b.lo == a.lo && b.hi == a.lo;
}

// The score of q . k in log2 units before the bias; in `slope` its derivative
// by z, 1 - tanh^2.  cap tanh(x) = cap - 2 cap / (e^2x + 1): right at both ends
// without a test, off by 2^-23 of the cap in the middle.
__device__ __forceinline__ float score(const Params& p, float dot, float* slope = nullptr) {
    if (p.cap2 == 0.f) {
        if (slope) *slope = 1.f;
        return dot * p.z_mul;
    }
    const float r = __builtin_amdgcn_rcpf(fast_exp2(dot * p.z_mul) + 1.f);
    if (slope) *slope = 4.f * r * (1.f - r);
    return __builtin_fmaf(-2.f * p.cap2, r, p.cap2);
}

// ---- tiles in LDS: rows of 32 DB channels and 16 bytes, which puts the rows
// that a wavefront reads at once into different banks ----

template <int DB>
struct Tile {
    static constexpr int CH = 32 * DB;       // channels, those behind a head's 0
    static constexpr int LD = CH * 2 + 16;   // bytes of a row
    static constexpr int VECS = 4 * DB;      // vectors of eight of a row
    static constexpr int BYTES = TILE * LD;
};

// Rows row0 + (lane % 32), channels 16 kk + 8 (lane / 32) ..: a product that
// contracts channels.
template <int DB>
__device__ __forceinline__ bf16x8 row_operand(const char* tile, int row0, int kk, int lane) {
    return *(const bf16x8*)(tile + (row0 + (lane & 31)) * Tile<DB>::LD + 32 * kk + 16 * (lane >> 5));
}

// Channel 32 mb + (lane % 32) of the 16 rows from row0, in the order of the
// scores' registers: a product that contracts rows.  Two transposing reads of
// four rows each for either half of the lanes.
template <int DB>
__device__ __forceinline__ bf16x8 column_operand(const char* tile, int row0, int mb, int lane) {
    typedef short s16x4 __attribute__((ext_vector_type(4)));
    typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
    const int row = row0 + 4 * (lane >> 5) + ((lane & 15) >> 2);
    const int at = 32 * mb + 16 * ((lane >> 4) & 1) + 4 * (lane & 3);
    const char* a = tile + row * Tile<DB>::LD + 2 * at;
    const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)a);
    const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(a + 8 * Tile<DB>::LD));
    const short __attribute__((ext_vector_type(8))) w = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
    return __builtin_bit_cast(bf16x8, w);
}

// Eight registers as an operand.
__device__ __forceinline__ bf16x8 packed(const float (&w)[16], int st) {
    bf16x8 o;
#pragma unroll
    for (int e = 0; e < 8; ++e) o[e] = f32_to_bf16(w[8 * st + e]);
    return o;
}

// acc += sum over the 32 rows from row0 of (their weights) x (their channels).
template <int DB>
__device__ __forceinline__ void add_rows(f32x16 (&acc)[DB], const float (&w)[16], const char* tile, int row0, int lane) {
#pragma unroll
    for (int st = 0; st < 2; ++st) {
        const bf16x8 b = packed(w, st);
#pragma unroll
        for (int mb = 0; mb < DB; ++mb)
            acc[mb] = mfma32x32x16(column_operand<DB>(tile, row0 + 16 * st, mb, lane), b, acc[mb]);
    }
}

// The eight values of an operand, infinities and NaN as 0.
__device__ __forceinline__ bf16x8 finite_only(bf16x8 v) {
    u32x4 w = __builtin_bit_cast(u32x4, v);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        if ((w[e] & 0x00007f80u) == 0x00007f80u) w[e] &= 0xffff0000u;
        if ((w[e] & 0x7f800000u) == 0x7f800000u) w[e] &= 0x0000ffffu;
    }
    return __builtin_bit_cast(bf16x8, w);
}

// The same where some weights are 0 because the mask hides the row, and the row
// may hold infinities or NaN: the product takes what is finite (bit for bit what
// it takes without them), and what is not goes to the weights that are not 0,
// value by value.
template <int DB>
__device__ __forceinline__ void add_rows_careful(f32x16 (&acc)[DB], const float (&w)[16], const char* tile, int row0,
                                                 int lane) {
#pragma unroll
    for (int st = 0; st < 2; ++st) {
        const bf16x8 b = packed(w, st);
#pragma unroll
        for (int mb = 0; mb < DB; ++mb)
            acc[mb] = mfma32x32x16(finite_only(column_operand<DB>(tile, row0 + 16 * st, mb, lane)), b, acc[mb]);
    }
#pragma unroll 1
    for (int j = 0; j < 32; ++j) {
        const int reg = 4 * (j >> 3) + (j & 3);
        float x = 0.f;
#pragma unroll
        for (int r = 0; r < 16; ++r) x = r == reg ? w[r] : x;
        x = __shfl(x, (lane & 31) + 32 * ((j >> 2) & 1));
#pragma unroll
        for (int mb = 0; mb < DB; ++mb)
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                const bf16x4 c = *(const bf16x4*)(tile + (row0 + j) * Tile<DB>::LD + 2 * (32 * mb + 8 * g + 4 * (lane >> 5)));
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float v = bf16_to_f32(c[e]), o = acc[mb][4 * g + e];
                    acc[mb][4 * g + e] = x != 0.f && !(fabsf(v) < INFINITY) ? __builtin_fmaf(x, v, o) : o;
                }
            }
    }
}

// Whether any lane of the wavefront holds a value that is no number.
template <int DB>
__device__ __forceinline__ bool any_not_finite(const f32x16 (&acc)[DB]) {
    bool bad = false;
#pragma unroll
    for (int mb = 0; mb < DB; ++mb)
#pragma unroll
        for (int r = 0; r < 16; ++r) bad |= !(fabsf(acc[mb][r]) < INFINITY);
    return __any(bad);
}

__device__ __forceinline__ float max_halves(float v) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float sum_halves(float v) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// The least and largest document of a wavefront's lanes, those out of play given as `in` false.
__device__ __forceinline__ DocRange range_of_lanes(int doc, bool in) {
    int lo = in ? doc : 0x7fffffff, hi = in ? doc : -1;
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) {
        lo = min(lo, __shfl_xor(lo, d));
        hi = max(hi, __shfl_xor(hi, d));
    }
    return DocRange{__builtin_amdgcn_readfirstlane(lo), __builtin_amdgcn_readfirstlane(hi)};
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

// f(head's channels in blocks of 32).
template <typename F>
hipError_t with_blocks(int head_dim, F f) {
    using std::integral_constant;
    switch ((head_dim + 31) / 32) {
        case 1: return f(integral_constant<int, 1>());
        case 2: return f(integral_constant<int, 2>());
        case 3: return f(integral_constant<int, 3>());
        default: return f(integral_constant<int, 4>());
    }
}

}  // namespace pcpp

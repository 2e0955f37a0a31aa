// Attention with masks, a bias by distance and capped scores: argument checks,
// workspace and launches.
//   pcpp_masked_attention(_workspace_size), pcpp_masked_attention_backward(_workspace_size)

#include <math.h>
#include <stdint.h>

#include <type_traits>

#include "../../include/pcpp.h"
#include "args.h"
#include "masked_attention.h"

#define PCPP_EXPORT extern "C" __attribute__((visibility("default")))

namespace pcpp {

using namespace masked;

namespace {

constexpr int kMaxTokens = 1 << 24;
constexpr float kMaxCap = 4096.f;  // (a capped score is off by up to 2^-23 of the cap)
constexpr int64_t kMaxBatch = (int64_t)1 << 40;  // elements
constexpr int64_t kMaxRow = 1 << 24;             // 64 rows are less than 2^32 bytes
constexpr int64_t kMaxHeadTokens = 1 << 29, kMaxHeadBlocks = 1 << 22;
constexpr int64_t kMaxGradTokens = 1 << 27;      // masked_delta: 16 threads to a query of a head

// A tensor's rows in elements: [batch, tokens, width] at `row` and `batch`.
struct Layout {
    int64_t row, batch;
    int64_t bytes(int B, int tokens, int width) const {
        return 2 * ((int64_t)(B - 1) * batch + (int64_t)(tokens - 1) * row + width);
    }
};

// The strides as given, or contiguous; false if they are not allowed.
bool layout_of(int64_t row, int64_t batch, int B, int tokens, int width, Layout* o) {
    if (row < 0 || batch < 0 || row > kMaxRow || batch > kMaxBatch / B || row % 8 != 0 || batch % 8 != 0)
        return false;
    o->row = row == 0 ? width : row;
    if (o->row < width) return false;
    o->batch = batch == 0 ? o->row * tokens : batch;
    return B == 1 || o->batch >= (int64_t)(tokens - 1) * o->row + width;
}

struct Shape {
    Layout q, k, v, y;
};

int check_geom(const pcpp_masked_geom_t* g, Shape* s) {
    if (!g || g->reserved != 0) return PCPP_EINVAL;
    if (g->batch < 1 || g->batch > 65535 || g->n_q < 1 || g->n_q > kMaxTokens || g->n_kv < 1 || g->n_kv > kMaxTokens)
        return PCPP_EINVAL;
    if (g->heads < 1 || g->heads > 1024 || g->kv_heads < 1 || g->heads % g->kv_heads != 0) return PCPP_EINVAL;
    if (g->causal != 0 && g->causal != 1) return PCPP_EINVAL;
    if (!isfinite(g->scale) || !(g->cap >= 0.f && g->cap <= kMaxCap)) return PCPP_EINVAL;
    if (g->cap > 0.f && !isfinite(g->scale / g->cap * 2.f * LOG2E)) return PCPP_EINVAL;
    if (g->head_dim < 8 || g->head_dim % 8 != 0 || g->head_dim > 128) return PCPP_ENOTSUP;
    // A launch has fewer than 2^32 threads: 256 for 128 tokens of a sequence's head.
    const int64_t heads = (int64_t)g->batch * g->heads, most = g->n_q > g->n_kv ? g->n_q : g->n_kv;
    if (heads * most > kMaxHeadTokens || heads * ((most + 127) / 128) > kMaxHeadBlocks) return PCPP_EINVAL;
    const int qw = g->heads * g->head_dim, kw = g->kv_heads * g->head_dim;
    if (!layout_of(g->q_row, g->q_batch, g->batch, g->n_q, qw, &s->q) ||
        !layout_of(g->k_row, g->k_batch, g->batch, g->n_kv, kw, &s->k) ||
        !layout_of(g->v_row, g->v_batch, g->batch, g->n_kv, kw, &s->v) ||
        !layout_of(g->y_row, g->y_batch, g->batch, g->n_q, qw, &s->y))
        return PCPP_EINVAL;
    return PCPP_OK;
}

int check_mask(const pcpp_masked_geom_t* g, const pcpp_mask_t* m) {
    if (!m) return PCPP_OK;
    const void* ptrs[] = {m->kv_len, m->q_pos, m->prefix, m->q_doc, m->kv_doc, m->slopes};
    for (const void* p : ptrs)
        if (!aligned_to(p, 4)) return PCPP_EINVAL;
    if ((m->q_doc == nullptr) != (m->kv_doc == nullptr) || (m->prefix && !g->causal)) return PCPP_EINVAL;
    return PCPP_OK;
}

int64_t round16(int64_t n) { return (n + 15) & ~(int64_t)15; }

int64_t range_bytes(const pcpp_masked_geom_t* g) {
    return round16((int64_t)g->batch * (tiles_of(g->n_q) + tiles_of(g->n_kv)) * sizeof(DocRange));
}

// Rows that share their keys few enough for masked_few: 64, or of all sequences
// as many as leave half the compute units without a workgroup of 32 rows, whose
// four wavefronts then share the keys (forward, us: 1000 queries and keys, 4
// heads of 64, 22 and 14; 4000, one of 128, 99 and 54; 500, 8 of 128, at the
// limit, 17.9 and 17.1; with twice the workgroups slower: 2000, 8 of 64, 39 and
// 45; so too where walks are short, 4 x 333, 16 of 64, causal, 14.4 and 18.2, or
// uneven, 2 x 4096, 10 of 64, 9 documents, 66 and 99).  How many pieces of the
// keys: as many as give every compute unit two workgroups, of eight tiles of 32
// keys or more (one token on up to 16384 keys, 64 groups: 80 us; with half as
// many pieces 98, with twice as many 95).
struct FewPlan {
    bool use;
    int pieces, row_blocks;
};
FewPlan few_plan(const pcpp_masked_geom_t* g) {
    const int64_t rows = (int64_t)g->heads / g->kv_heads * g->n_q, row_blocks = (rows + MASKED_FEW_ROWS - 1) / MASKED_FEW_ROWS;
    const int64_t groups = (int64_t)g->batch * g->kv_heads * row_blocks, tiles = (g->n_kv + 31) / 32;
    FewPlan f = {rows <= 2 * MASKED_FEW_ROWS || (groups <= 128 && g->n_kv >= 128), 1, (int)row_blocks};
    if (!f.use) return f;
    int64_t pieces = (512 + groups - 1) / groups;
    if (pieces > tiles / 8) pieces = tiles / 8;
    f.pieces = (int)(pieces > 0 ? pieces : 1);
    return f;
}
int64_t few_blocks(const pcpp_masked_geom_t* g, const FewPlan& f) {
    return f.use && f.pieces > 1 ? (int64_t)g->batch * g->kv_heads * f.row_blocks * f.pieces : 0;
}
int64_t few_floats(const pcpp_masked_geom_t* g) { return (int64_t)MASKED_FEW_ROWS * (32 * blocks_of(g->head_dim)); }

int64_t forward_bytes(const pcpp_masked_geom_t* g) {
    return range_bytes(g) + few_blocks(g, few_plan(g)) * (few_floats(g) + 2 * MASKED_FEW_ROWS) * 4;
}
int64_t delta_bytes(const pcpp_masked_geom_t* g) { return round16((int64_t)g->batch * g->heads * g->n_q * 4); }
// Pieces of the queries (of all heads) for the keys' gradients: with fewer
// blocks of keys than two to a compute unit (causal, of uneven length: four), as
// many as fill them, of two tiles of 64 queries or more (dk and dv with eight or
// more, and with two: 434 queries and keys, 4 heads of 128, 39 and 21 us; 1000
// causal, 8 heads on 2, 47 and 38).
int kv_pieces(const pcpp_masked_geom_t* g) {
    const int64_t blocks = (int64_t)g->batch * g->kv_heads * ((g->n_kv + 127) / 128);
    const int64_t tiles = (int64_t)g->heads / g->kv_heads * ((g->n_q + 63) / 64);
    int64_t n = ((g->causal ? 1024 : 512) + blocks - 1) / blocks;
    if (n > tiles / 2) n = tiles / 2;
    return (int)(n < 1 ? 1 : n);
}
int64_t kv_bytes(const pcpp_masked_geom_t* g) {
    const int n = kv_pieces(g);
    return n == 1 ? 0 : (int64_t)n * g->batch * g->kv_heads * g->n_kv * 2 * (32 * blocks_of(g->head_dim)) * 4;
}
int64_t backward_bytes(const pcpp_masked_geom_t* g) { return range_bytes(g) + 2 * delta_bytes(g) + kv_bytes(g); }

Params params_of(const pcpp_masked_geom_t* g, const pcpp_mask_t* m, const Shape& s, void* workspace) {
    Params p = {};
    p.q_row = s.q.row, p.k_row = s.k.row, p.v_row = s.v.row, p.y_row = s.y.row;
    p.q_batch = s.q.batch, p.k_batch = s.k.batch, p.v_batch = s.v.batch, p.y_batch = s.y.batch;
    p.B = g->batch, p.nq = g->n_q, p.nkv = g->n_kv, p.H = g->heads, p.KH = g->kv_heads, p.G = g->heads / g->kv_heads;
    p.D = g->head_dim;
    p.causal = g->causal;
    p.scale = g->scale;
    p.cap = g->cap;
    p.cap2 = g->cap * LOG2E;
    p.z_mul = g->cap > 0.f ? g->scale / g->cap * 2.f * LOG2E : g->scale * LOG2E;
    if (m) {
        p.kv_len = m->kv_len, p.q_pos = m->q_pos, p.prefix = m->prefix;
        p.q_doc = m->q_doc, p.kv_doc = m->kv_doc, p.slopes = m->slopes;
    }
    p.q_range = (DocRange*)workspace;
    p.kv_range = p.q_range + (int64_t)g->batch * tiles_of(g->n_q);
    return p;
}

// The mask's arrays as inputs.
int mask_ranges(const pcpp_masked_geom_t* g, const pcpp_mask_t* m, Range* o) {
    if (!m) return 0;
    const int64_t b = 4 * (int64_t)g->batch;
    o[0] = {m->kv_len, b}, o[1] = {m->q_pos, b}, o[2] = {m->prefix, b};
    o[3] = {m->q_doc, b * g->n_q}, o[4] = {m->kv_doc, b * g->n_kv}, o[5] = {m->slopes, 4 * (int64_t)g->heads};
    return 6;
}

}  // namespace

}  // namespace pcpp

using namespace pcpp;

PCPP_EXPORT size_t pcpp_masked_attention_workspace_size(const pcpp_masked_geom_t* g) {
    Shape s;
    return check_geom(g, &s) == PCPP_OK ? (size_t)forward_bytes(g) : 0;
}

PCPP_EXPORT int pcpp_masked_attention(const pcpp_masked_geom_t* g, const pcpp_mask_t* m, const void* q, const void* k,
                                      const void* v, void* y, float* lse, void* workspace, size_t ws_bytes,
                                      void* stream) {
    Shape sh;
    int st = check_geom(g, &sh);
    if (st == PCPP_OK) st = check_mask(g, m);
    if (st != PCPP_OK) return st;
    const void* ptrs[] = {q, k, v, y};
    for (const void* a : ptrs)
        if (!a || !aligned_to(a, 16)) return PCPP_EINVAL;
    if (!aligned_to(lse, 4)) return PCPP_EINVAL;
    const int64_t need = forward_bytes(g);
    if (!workspace || ws_bytes < (size_t)need) return PCPP_EWORKSPACE;
    if (!aligned_to(workspace, 16)) return PCPP_EINVAL;
    const int qw = g->heads * g->head_dim, kw = g->kv_heads * g->head_dim;
    const Range out[] = {{y, sh.y.bytes(g->batch, g->n_q, qw)}, {lse, 4 * (int64_t)g->batch * g->heads * g->n_q}, {workspace, need}};
    Range in[9] = {{q, sh.q.bytes(g->batch, g->n_q, qw)}, {k, sh.k.bytes(g->batch, g->n_kv, kw)}, {v, sh.v.bytes(g->batch, g->n_kv, kw)}};
    if (outputs_overlap(out, 3, in, 3 + mask_ranges(g, m, in + 3))) return PCPP_EINVAL;
    Params p = params_of(g, m, sh, workspace);
    p.q = (const bf16*)q, p.k = (const bf16*)k, p.v = (const bf16*)v, p.y = (bf16*)y;
    p.lse = lse;
    const hipStream_t s = (hipStream_t)stream;
    if (p.kv_doc && launch_masked_ranges(p, s) != hipSuccess) return PCPP_EHIP;
    const FewPlan f = few_plan(g);
    if (!f.use) return launch_masked_forward(p, s) == hipSuccess ? PCPP_OK : PCPP_EHIP;
    p.pieces = f.pieces;
    p.row_blocks = f.row_blocks;
    p.part_o = (float*)((char*)workspace + range_bytes(g));
    p.part_ml = p.part_o + few_blocks(g, f) * few_floats(g);
    return launch_masked_few(p, s) == hipSuccess ? PCPP_OK : PCPP_EHIP;
}

static int check_backward(const pcpp_masked_geom_t* g, Shape* s) {
    const int st = check_geom(g, s);
    return st == PCPP_OK && (int64_t)g->batch * g->heads * g->n_q > kMaxGradTokens ? PCPP_EINVAL : st;
}

PCPP_EXPORT size_t pcpp_masked_attention_backward_workspace_size(const pcpp_masked_geom_t* g) {
    Shape s;
    return check_backward(g, &s) == PCPP_OK ? (size_t)backward_bytes(g) : 0;
}

PCPP_EXPORT int pcpp_masked_attention_backward(const pcpp_masked_geom_t* g, const pcpp_mask_t* m, const void* q,
                                               const void* k, const void* v, const void* y, const float* lse,
                                               const void* dy, void* dq, void* dk, void* dv, void* workspace,
                                               size_t ws_bytes, void* stream) {
    Shape sh;
    int st = check_backward(g, &sh);
    if (st == PCPP_OK) st = check_mask(g, m);
    if (st != PCPP_OK) return st;
    const void* needed[] = {q, k, v, y, lse, dy};
    for (const void* a : needed)
        if (!a) return PCPP_EINVAL;
    const void* ptrs[] = {q, k, v, y, dy, dq, dk, dv};
    for (const void* a : ptrs)
        if (!aligned_to(a, 16)) return PCPP_EINVAL;
    if (!aligned_to(lse, 4) || (!dq && !dk) || (dk == nullptr) != (dv == nullptr)) return PCPP_EINVAL;
    const int64_t need = backward_bytes(g);
    if (!workspace || ws_bytes < (size_t)need) return PCPP_EWORKSPACE;
    if (!aligned_to(workspace, 16)) return PCPP_EINVAL;
    const int qw = g->heads * g->head_dim, kw = g->kv_heads * g->head_dim;
    const int64_t qb = sh.q.bytes(g->batch, g->n_q, qw), kb = sh.k.bytes(g->batch, g->n_kv, kw);
    const int64_t vb = sh.v.bytes(g->batch, g->n_kv, kw), yb = sh.y.bytes(g->batch, g->n_q, qw);
    // The gradients may lie in each other's rows, as q, k and v of one product
    // do: each is held against the inputs, and the workspace, alone.
    Range in[13] = {{q, qb}, {k, kb}, {v, vb}, {y, yb}, {dy, yb}, {lse, 4 * (int64_t)g->batch * g->heads * g->n_q}, {workspace, need}};
    const int n_in = 7 + mask_ranges(g, m, in + 7);
    const Range out[] = {{dq, qb}, {dk, kb}, {dv, vb}};
    for (const Range& o : out)
        if (outputs_overlap(&o, 1, in, n_in)) return PCPP_EINVAL;
    if (dk && (dq == dk || dq == dv || dk == dv)) return PCPP_EINVAL;
    if (outputs_overlap(&in[6], 1, in, 6) || outputs_overlap(&in[6], 1, in + 7, n_in - 7)) return PCPP_EINVAL;
    Params p = params_of(g, m, sh, workspace);
    p.q = (const bf16*)q, p.k = (const bf16*)k, p.v = (const bf16*)v, p.y = (bf16*)y, p.dy = (const bf16*)dy;
    p.lse = (float*)lse;
    p.dq = (bf16*)dq, p.dk = (bf16*)dk, p.dv = (bf16*)dv;
    p.delta = (float*)((char*)workspace + range_bytes(g));
    p.lse2 = (float*)((char*)p.delta + delta_bytes(g));
    p.part_o = (float*)((char*)p.lse2 + delta_bytes(g));
    p.pieces = kv_pieces(g);
    const hipStream_t s = (hipStream_t)stream;
    if (p.kv_doc && launch_masked_ranges(p, s) != hipSuccess) return PCPP_EHIP;
    if (launch_masked_delta(p, s) != hipSuccess) return PCPP_EHIP;
    if (launch_masked_dq(p, s) != hipSuccess) return PCPP_EHIP;  // dq, if wanted, and delta for what follows
    if (dk && launch_masked_dkv(p, s) != hipSuccess) return PCPP_EHIP;
    return PCPP_OK;
}

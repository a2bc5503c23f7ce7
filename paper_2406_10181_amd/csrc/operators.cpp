// extern "C" entry points of the operators of a training step: attention, residual norm, dropout.  Argument checks, workspace carving, launches.
#include <algorithm>
#include <cmath>

#include "operator_checks.h"
#include "residual_norm.h"

namespace lsp {

hipError_t launch_dropout(const void* x, void* y, int64_t rows, int64_t width, const Dropout& drop, lsp_dtype dtype, hipStream_t st);

template <typename D> hipError_t attention_forward_of(const AttentionArgs& a, hipStream_t st);
template <typename D> hipError_t attention_backward_of(const AttentionArgs& a, hipStream_t st);

hipError_t launch_attention_forward(const AttentionArgs& a, lsp_dtype dtype, hipStream_t st) {
    return dtype == LSP_F32 ? attention_forward_of<F32>(a, st) : dtype == LSP_F16 ? attention_forward_of<F16>(a, st) : attention_forward_of<BF16>(a, st);
}
hipError_t launch_attention_backward(const AttentionArgs& a, lsp_dtype dtype, hipStream_t st) {
    return dtype == LSP_F32 ? attention_backward_of<F32>(a, st) : dtype == LSP_F16 ? attention_backward_of<F16>(a, st) : attention_backward_of<BF16>(a, st);
}

size_t attention_partial_bytes(const AttentionArgs& a) {
    if (a.splits <= 1) return 0;
    return align_up((size_t)a.splits * a.batch * a.heads * a.q_len * ((size_t)a.head_dim + 2) * sizeof(float), 256);
}

// Eight waves a workgroup for wide heads and long texts, where that leaves every CU a workgroup: a tile of keys serves twice the queries.  16 heads of 128, one text of
// 8192, bf16: 266 us, with four waves 282; 32 heads, four texts of 1024: 51.5 both; 16 heads of 64, eight texts of 2048: 187 and 179; padded texts of 777: 39 and 29.
static int waves_for(int64_t units, int64_t rows, int64_t keys, int head_dim, lsp_dtype dtype) {
    return dtype != LSP_F32 && head_dim > 64 && keys >= 2048 && units * ((rows + 8 * kWaveRows - 1) / (8 * kWaveRows)) >= 256 ? 8 : 4;
}

// In how many parts the steps of a tile are done, by workgroups of their own: what takes the least time by a rough account.  A step takes a workgroup that has a CU for itself about
// step_us; a part's sums (`bytes` for all tiles) are written and read again, at 5 TB/s, and are added by a launch of its own, 4 us.  No more parts than run at once: two
// workgroups a CU, in the backward pass of fp32 beyond heads of 32 one (4 texts of 512, 8 heads of 64: 129 us, with parts for two 143; 2 of 1024, 16 heads of 128: 441 and 461).
// Against parts of four steps or more, as many as give each CU two workgroups, forward and backward kernels: fp32, one text of 469, 2 heads of 128, 97 us, so 62; bf16, three texts of
// 407, 1 head of 128, 41 and 35; fp16, two texts of 1000, 8 heads of 64, 64 and 57; one text of 1464, 8 heads of 128, 104 and 102; but bf16, one text of 4691, 2 heads, 130 and 133.
static int parts_for(int64_t tiles, int64_t steps, double step_us, int64_t bytes, int at_once = 512) {
    const int64_t most = std::min<int64_t>({at_once / std::max<int64_t>(tiles, 1), steps, 16});
    int best = 1;
    double least = (double)steps * step_us;
    for (int p = 2; p <= most; ++p) {
        const double us = (double)((steps + p - 1) / p) * step_us + 4.0 + p * (0.25 + 2.0 * (double)bytes / 5e6);
        if (us < least) { least = us; best = p; }
    }
    return best;
}
// of a wave's 32 rows and one tile of the others, `products` of them; 16 bits: 64 a tile, fp32: 32
static double step_us(const AttentionArgs& a, lsp_dtype dtype, int products) {
    const int dim = (a.head_dim + 31) / 32 * 32;
    return products * dim * (dtype == LSP_F32 ? 1.0 / 64 : 1.0 / 256) * (a.drop.limit ? 1.5 : 1.0);
}

void plan_attention_forward(AttentionArgs& a, lsp_dtype dtype) {
    // Few queries: the query heads that share a key head go into one tile of rows, so that keys and values are read once for all of them.
    // (Its rows are addressed with 32 bits from the first head's first row.)
    a.packed = a.group > 1 && (int64_t)a.group * a.q_len <= 4 * kWaveRows && ((int64_t)a.group * a.q.head + (int64_t)a.q_len * a.q.position) * 4 < ((int64_t)1 << 31);
    a.rows = a.packed ? a.group * a.q_len : a.q_len;
    const int64_t units = (int64_t)a.batch * (a.packed ? a.kv_heads : a.heads);
    a.few = dtype != LSP_F32 && a.rows <= 32 && a.drop.limit == 0;
    a.waves = a.packed ? 4 : waves_for(units, a.rows, a.k_len, a.head_dim, dtype);
    a.tiles = a.few ? 1 : (int)((a.rows + a.waves * kWaveRows - 1) / (a.waves * kWaveRows));
    // Few tiles of rows: the keys are split.  (Few queries: as far as that gives each CU four workgroups, and each of these two tiles of keys a wave.)
    const int tile = a.few ? 32 : tile_rows_of(dtype);
    const int64_t row_tiles = units * a.tiles;
    const int key_tiles = (a.k_len + tile - 1) / tile;
    const int splits = a.few ? (int)std::min<int64_t>({std::max<int64_t>(1024 / row_tiles, 1), std::max(key_tiles / 8, 1), 64})
                     : a.waves == 8 ? 1 : parts_for(row_tiles, key_tiles, step_us(a, dtype, 2), units * a.rows * a.head_dim * 4);
    a.split_tiles = (key_tiles + splits - 1) / splits;
    a.splits = (key_tiles + a.split_tiles - 1) / a.split_tiles;
}

void plan_attention_backward(AttentionArgs& a, lsp_dtype dtype) {
    const int64_t key_tiles = (int64_t)a.batch * a.kv_heads * ((a.k_len + kBackwardRows - 1) / kBackwardRows);
    const int64_t query_tiles = (int64_t)a.batch * a.heads * ((a.q_len + kBackwardRows - 1) / kBackwardRows);
    const int64_t q_steps = (a.q_len + tile_rows_of(dtype) - 1) / tile_rows_of(dtype), k_steps = (a.k_len + tile_rows_of(dtype) - 1) / tile_rows_of(dtype);
    const int at_once = dtype == LSP_F32 && a.head_dim > 32 ? 256 : 512;
    a.key_parts = parts_for(key_tiles, a.group * q_steps, step_us(a, dtype, 4), (int64_t)8 * a.batch * a.kv_heads * a.k_len * a.head_dim, at_once);
    a.query_parts = parts_for(query_tiles, k_steps, step_us(a, dtype, 3), (int64_t)4 * a.batch * a.heads * a.q_len * a.head_dim, at_once);
}
size_t attention_backward_partial_bytes(const AttentionArgs& a) {
    const size_t keys = a.key_parts > 1 ? (size_t)2 * a.key_parts * a.batch * a.kv_heads * a.k_len : 0;
    const size_t queries = a.query_parts > 1 ? (size_t)a.query_parts * a.batch * a.heads * a.q_len : 0;
    return align_up((keys + queries) * a.head_dim * sizeof(float), 256);
}

}  // namespace lsp

namespace {

constexpr float kLog2e = 1.44269504088896341f;

int check_attention_shape(const lsp_attention_problem* p, lsp_dtype t) {
    if (!p) return LSP_ERR_NULL;
    if (p->batch <= 0 || p->heads <= 0 || p->kv_heads <= 0 || p->q_len <= 0 || p->k_len <= 0 || p->head_dim <= 0) return LSP_ERR_SHAPE;
    if (p->heads % p->kv_heads || p->head_dim % 8 || p->head_dim > LSP_MAX_HEAD_DIM) return LSP_ERR_SHAPE;
    if (p->q_len > (1 << 30) || p->k_len > (1 << 30) || (p->causal != 0 && p->causal != 1)) return LSP_ERR_SHAPE;
    // a launch has fewer than 2^32 threads: 16 for every row of dO and of V, where delta is made (the others: launches())
    if ((int64_t)p->batch * p->heads > (1 << 24) || (int64_t)p->batch * p->heads * std::max(p->q_len, p->k_len) >= ((int64_t)1 << 27)) return LSP_ERR_SHAPE;
    if (!known(t)) return LSP_ERR_DTYPE;
    return LSP_OK;
}

int check_attention(const lsp_attention_problem* p, lsp_dtype t) {
    if (!p || !p->Q || !p->K || !p->V || !p->O || !p->L) return LSP_ERR_NULL;
    int rc = check_attention_shape(p, t);
    if (rc != LSP_OK) return rc;
    if (!rate(p->dropout) || !(p->scale > 0.0f) || !std::isfinite(p->scale * kLog2e)) return LSP_ERR_VALUE;
    if ((rc = check_strides(p->q_stride, p->batch, p->q_len, p->heads, p->head_dim, t, false)) != LSP_OK) return rc;
    if ((rc = check_strides(p->k_stride, p->batch, p->k_len, p->kv_heads, p->head_dim, t, false)) != LSP_OK) return rc;
    if ((rc = check_strides(p->v_stride, p->batch, p->k_len, p->kv_heads, p->head_dim, t, false)) != LSP_OK) return rc;
    if ((rc = check_strides(p->o_stride, p->batch, p->q_len, p->heads, p->head_dim, t, true)) != LSP_OK) return rc;
    if (!aligned16(p->Q) || !aligned16(p->K) || !aligned16(p->V) || !aligned16(p->O) || !aligned16(p->L)) return LSP_ERR_ALIGN;
    if ((reinterpret_cast<uintptr_t>(p->q_lens) | reinterpret_cast<uintptr_t>(p->k_lens)) & 3u) return LSP_ERR_ALIGN;
    return LSP_OK;
}

lsp::AttentionArgs attention_args(const lsp_attention_problem* p) {
    lsp::AttentionArgs a{};
    a.q = strided(p->Q, p->q_stride, p->batch, p->q_len, p->heads);
    a.k = strided(p->K, p->k_stride, p->batch, p->k_len, p->kv_heads);
    a.v = strided(p->V, p->v_stride, p->batch, p->k_len, p->kv_heads);
    a.o = strided(p->O, p->o_stride, p->batch, p->q_len, p->heads);
    a.L = p->L;
    a.q_lens = p->q_lens; a.k_lens = p->k_lens;
    a.batch = p->batch; a.heads = p->heads; a.kv_heads = p->kv_heads; a.group = p->heads / p->kv_heads;
    a.q_len = p->q_len; a.k_len = p->k_len; a.head_dim = p->head_dim; a.causal = p->causal;
    a.scale = p->scale; a.scale_log2 = p->scale * kLog2e;
    a.drop = lsp::make_dropout(p->dropout, p->seed, p->offset);
    return a;
}

// Whether the workgroups of the plan have fewer than 2^32 threads; the backward pass has those for queries and those for keys in one launch.
bool launches_forward(const lsp::AttentionArgs& a) {
    return (int64_t)a.batch * (a.packed ? a.kv_heads : a.heads) * a.tiles * a.splits * a.waves * 64 < ((int64_t)1 << 32);
}
bool launches_backward(const lsp::AttentionArgs& a) {
    const auto tiles = [](int64_t positions) { return (positions + lsp::kBackwardRows - 1) / lsp::kBackwardRows; };
    return (a.batch * (int64_t)a.heads * tiles(a.q_len) * a.query_parts + a.batch * (int64_t)a.kv_heads * tiles(a.k_len) * a.key_parts) * 256 < ((int64_t)1 << 32);
}

constexpr size_t kNormBytes = 2 * lsp::kNormSlots * sizeof(float);
size_t delta_bytes(const lsp_attention_problem* p) { return lsp::align_up((size_t)p->batch * p->heads * p->q_len * sizeof(float), 256); }

int check_norm_shape(const lsp_residual_norm_problem* p, lsp_dtype t) {
    if (!p) return LSP_ERR_NULL;
    if (p->rows <= 0 || p->rows > LSP_MAX_ROWS || p->width <= 0 || p->width > LSP_MAX_WIDTH || !norm_kind(p->post) || !norm_kind(p->pre)) return LSP_ERR_SHAPE;
    if (!known(t)) return LSP_ERR_DTYPE;
    return LSP_OK;
}

int check_norm(const lsp_residual_norm_problem* p, lsp_dtype t) {
    if (!p || !p->x || !p->f || !p->y || !p->stats || (!p->h && p->pre != LSP_NORM_NONE)) return LSP_ERR_NULL;
    const int rc = check_norm_shape(p, t);
    if (rc != LSP_OK) return rc;
    if (!rate(p->dropout) || !std::isfinite(p->residual_scale) || !std::isfinite(p->branch_scale) || !(p->eps >= 0.0f) || !std::isfinite(p->eps)) return LSP_ERR_VALUE;
    const int64_t most = (int64_t)1 << 40;
    for (const int64_t s : {p->x_stride, p->f_stride, p->y_stride, p->h ? p->h_stride : p->width})
        if (p->rows > 1 && (s < p->width || s > most)) return LSP_ERR_SHAPE;
    for (const void* q : {p->x, p->f, static_cast<const void*>(p->y), static_cast<const void*>(p->h), static_cast<const void*>(p->stats), p->post_weight, p->post_bias, p->gate,
                          p->pre_weight, p->pre_bias})
        if (!aligned16(q)) return LSP_ERR_ALIGN;
    if (!on_it(p->x, p->x_stride, p->y, p->y_stride, p->rows) || !on_it(p->f, p->f_stride, p->y, p->y_stride, p->rows)) return LSP_ERR_SHAPE;
    if (p->h && (!on_it(p->x, p->x_stride, p->h, p->h_stride, p->rows) || !on_it(p->f, p->f_stride, p->h, p->h_stride, p->rows) || !on_it(p->y, p->y_stride, p->h, p->h_stride, p->rows)))
        return LSP_ERR_SHAPE;
    return LSP_OK;
}

lsp::ResidualNormArgs norm_args(const lsp_residual_norm_problem* p) {
    lsp::ResidualNormArgs a{};
    a.x = p->x; a.f = p->f; a.y = p->y; a.h = p->h; a.stats = p->stats;
    a.post_w = p->post_weight; a.post_b = p->post_bias; a.gate = p->gate; a.pre_w = p->pre_weight; a.pre_b = p->pre_bias;
    a.x_stride = p->x_stride; a.f_stride = p->f_stride; a.y_stride = p->y_stride; a.h_stride = p->h_stride;
    a.rows = p->rows; a.width = p->width; a.post = p->post; a.pre = p->pre;
    a.eps = p->eps; a.residual_scale = p->residual_scale; a.branch_scale = p->branch_scale;
    a.drop = lsp::make_dropout(p->dropout, p->seed, p->offset);
    return a;
}

}  // namespace

extern "C" {

int lsp_dropout(const void* x, void* y, int64_t rows, int64_t width, float dropout, uint64_t seed, uint32_t offset, lsp_dtype dtype, void* stream) {
    if (!x || !y) return LSP_ERR_NULL;
    if (rows <= 0 || width <= 0 || width > INT32_MAX - 7 || rows > ((int64_t)1 << 31) / ((width + 7) / 8)) return LSP_ERR_SHAPE;   // a thread for every block of eight
    if (!known(dtype)) return LSP_ERR_DTYPE;
    if (!rate(dropout)) return LSP_ERR_VALUE;
    if (!aligned16(x) || !aligned16(y)) return LSP_ERR_ALIGN;
    return done(lsp::launch_dropout(x, y, rows, width, lsp::make_dropout(dropout, seed, offset), dtype, static_cast<hipStream_t>(stream)));
}

size_t lsp_attention_forward_workspace_bytes(const lsp_attention_problem* p, lsp_dtype dtype) {
    if (check_attention_shape(p, dtype) != LSP_OK) return 0;
    lsp::AttentionArgs a = attention_args(p);
    lsp::plan_attention_forward(a, dtype);
    return launches_forward(a) ? lsp::attention_partial_bytes(a) : 0;
}

int lsp_attention_forward(const lsp_attention_problem* p, lsp_dtype dtype, void* workspace, size_t workspace_bytes, void* stream) {
    const int rc = check_attention(p, dtype);
    if (rc != LSP_OK) return rc;
    lsp::AttentionArgs a = attention_args(p);
    lsp::plan_attention_forward(a, dtype);
    if (!launches_forward(a)) return LSP_ERR_SHAPE;
    const size_t need = lsp::attention_partial_bytes(a);
    if (need && (!workspace || workspace_bytes < need || !aligned16(workspace))) return LSP_ERR_WORKSPACE;
    a.partial = static_cast<float*>(workspace);
    return done(lsp::launch_attention_forward(a, dtype, static_cast<hipStream_t>(stream)));
}

// delta | norms | parts
size_t lsp_attention_backward_workspace_bytes(const lsp_attention_problem* p, lsp_dtype dtype) {
    if (check_attention_shape(p, dtype) != LSP_OK) return 0;
    lsp::AttentionArgs a = attention_args(p);
    lsp::plan_attention_backward(a, dtype);
    return launches_backward(a) ? delta_bytes(p) + kNormBytes + lsp::attention_backward_partial_bytes(a) : 0;
}

int lsp_attention_backward(const lsp_attention_problem* p, const lsp_attention_gradients* g, lsp_dtype dtype, void* workspace, size_t workspace_bytes, void* stream) {
    if (!p || !g || !g->dO || !g->dQ || !g->dK || !g->dV) return LSP_ERR_NULL;
    int rc = check_attention(p, dtype);
    if (rc != LSP_OK) return rc;
    if ((rc = check_strides(g->do_stride, p->batch, p->q_len, p->heads, p->head_dim, dtype, false)) != LSP_OK) return rc;
    if ((rc = check_strides(g->dq_stride, p->batch, p->q_len, p->heads, p->head_dim, dtype, true)) != LSP_OK) return rc;
    if ((rc = check_strides(g->dk_stride, p->batch, p->k_len, p->kv_heads, p->head_dim, dtype, true)) != LSP_OK) return rc;
    if ((rc = check_strides(g->dv_stride, p->batch, p->k_len, p->kv_heads, p->head_dim, dtype, true)) != LSP_OK) return rc;
    if (!aligned16(g->dO) || !aligned16(g->dQ) || !aligned16(g->dK) || !aligned16(g->dV)) return LSP_ERR_ALIGN;
    const size_t need = lsp_attention_backward_workspace_bytes(p, dtype);
    if (!need) return LSP_ERR_SHAPE;                                      // (a launch too large)
    if (!workspace || workspace_bytes < need || !aligned16(workspace)) return LSP_ERR_WORKSPACE;
    lsp::AttentionArgs a = attention_args(p);
    a.d_o = strided(g->dO, g->do_stride, p->batch, p->q_len, p->heads);
    a.dq = strided(g->dQ, g->dq_stride, p->batch, p->q_len, p->heads);
    a.dk = strided(g->dK, g->dk_stride, p->batch, p->k_len, p->kv_heads);
    a.dv = strided(g->dV, g->dv_stride, p->batch, p->k_len, p->kv_heads);
    a.delta = static_cast<float*>(workspace);
    a.norms = reinterpret_cast<float*>(static_cast<uint8_t*>(workspace) + delta_bytes(p));
    a.partial = reinterpret_cast<float*>(static_cast<uint8_t*>(workspace) + delta_bytes(p) + kNormBytes);
    lsp::plan_attention_backward(a, dtype);
    return done(lsp::launch_attention_backward(a, dtype, static_cast<hipStream_t>(stream)));
}

int lsp_residual_norm_forward(const lsp_residual_norm_problem* p, lsp_dtype dtype, void* stream) {
    const int rc = check_norm(p, dtype);
    if (rc != LSP_OK) return rc;
    return done(lsp::launch_residual_norm_forward(norm_args(p), dtype, static_cast<hipStream_t>(stream)));
}

size_t lsp_residual_norm_backward_workspace_bytes(const lsp_residual_norm_problem* p, lsp_dtype dtype) {
    if (check_norm_shape(p, dtype) != LSP_OK) return 0;
    return lsp::residual_norm_partial_bytes(p->rows, p->width);
}

int lsp_residual_norm_backward(const lsp_residual_norm_problem* p, const lsp_residual_norm_gradients* g, lsp_dtype dtype, void* workspace, size_t workspace_bytes, void* stream) {
    if (!p || !g || !g->dy || !g->dx || !g->df || (!g->dh && p->pre != LSP_NORM_NONE)) return LSP_ERR_NULL;
    const int rc = check_norm(p, dtype);
    if (rc != LSP_OK) return rc;
    if (p->y == p->x) return LSP_ERR_SHAPE;                              // x is needed as it was
    const int64_t most = (int64_t)1 << 40;
    for (const int64_t s : {g->dy_stride, g->dx_stride, g->df_stride, g->dh ? g->dh_stride : p->width})
        if (p->rows > 1 && (s < p->width || s > most)) return LSP_ERR_SHAPE;
    for (const void* q : {g->dy, g->dh, static_cast<const void*>(g->dx), static_cast<const void*>(g->df)})
        if (!aligned16(q)) return LSP_ERR_ALIGN;
    for (const float* q : {g->post_weight, g->post_bias, g->gate, g->pre_weight, g->pre_bias})
        if (!aligned16(q)) return LSP_ERR_ALIGN;
    const struct { const void* at; int64_t stride; } in[4] = {{p->x, p->x_stride}, {p->f, p->f_stride}, {g->dy, g->dy_stride}, {g->dh, g->dh_stride}};
    for (const auto& i : in)
        if (!on_it(i.at, i.stride, g->dx, g->dx_stride, p->rows) || !on_it(i.at, i.stride, g->df, g->df_stride, p->rows)) return LSP_ERR_SHAPE;
    if (!on_it(g->dx, g->dx_stride, g->df, g->df_stride, p->rows)) return LSP_ERR_SHAPE;
    const size_t need = lsp_residual_norm_backward_workspace_bytes(p, dtype);
    if (!workspace || workspace_bytes < need || !aligned16(workspace)) return LSP_ERR_WORKSPACE;
    if (p->y == p->f || (p->h && (p->h == p->x || p->h == p->f))) return LSP_ERR_SHAPE;      // as are x and f
    lsp::ResidualNormArgs a = norm_args(p);
    a.dy = g->dy; a.dh = g->dh; a.dx = g->dx; a.df = g->df;
    a.dy_stride = g->dy_stride; a.dh_stride = g->dh_stride; a.dx_stride = g->dx_stride; a.df_stride = g->df_stride;
    a.grads[0] = g->pre_weight; a.grads[1] = g->pre_bias; a.grads[2] = g->gate; a.grads[3] = g->post_weight; a.grads[4] = g->post_bias;
    if (p->pre == LSP_NORM_NONE && (g->pre_weight || g->pre_bias)) return LSP_ERR_SHAPE;      // a norm that is none has no weights
    if (p->post == LSP_NORM_NONE && (g->post_weight || g->post_bias)) return LSP_ERR_SHAPE;
    a.partial = static_cast<float*>(workspace);
    return done(lsp::launch_residual_norm_backward(a, dtype, static_cast<hipStream_t>(stream)));
}

}  // extern "C"

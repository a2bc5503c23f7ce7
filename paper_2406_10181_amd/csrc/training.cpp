// extern "C" entry points of what a training step needs around attention: rotary positions with norms of the heads, cross entropy, AdamW.  Argument checks, workspace carving,
// launches.
#include <cfloat>

#include "adamw.h"
#include "cross_entropy.h"
#include "operator_checks.h"
#include "rotary.h"

namespace {

constexpr int64_t kMostLaunch = (int64_t)1 << 24;                        // workgroups of 256 threads: fewer than 2^32 threads

int check_rotary_shape(const lsp_rotary_problem* p, lsp_dtype t) {
    if (!p) return LSP_ERR_NULL;
    if (p->batch <= 0 || p->length <= 0 || p->cache <= 0 || p->heads <= 0 || p->kv_heads <= 0 || p->head_dim <= 0 || p->rotated < 0) return LSP_ERR_SHAPE;
    if (p->head_dim % 8 || p->head_dim > LSP_MAX_HEAD_DIM || p->rotated % 8 || p->rotated > p->head_dim) return LSP_ERR_SHAPE;
    if ((p->neighbours != 0 && p->neighbours != 1) || !norm_kind(p->norm)) return LSP_ERR_SHAPE;
    const int64_t most = (int64_t)1 << 31, rows = (int64_t)p->heads + 2 * (int64_t)p->kv_heads, tokens = (int64_t)p->batch * p->length;
    if (rows >= most || tokens >= most || rows * tokens >= most || (int64_t)p->batch * p->cache >= most) return LSP_ERR_SHAPE;
    if (!known(t)) return LSP_ERR_DTYPE;
    return LSP_OK;
}

// One operand's strides: as in attention, and heads less than 256 MiB apart (16 of them are addressed with 32 bits)
int check_heads(const int64_t (&s)[3], int64_t batch, int64_t positions, int64_t heads, int32_t dim, lsp_dtype t, bool written) {
    const int rc = check_strides(s, batch, positions, heads, dim, t, written);
    return rc == LSP_OK && heads > 1 && s[2] * elem_size(t) >= ((int64_t)1 << 28) ? LSP_ERR_SHAPE : rc;
}
bool same_strides(const int64_t (&a)[3], const int64_t (&b)[3], int64_t batch, int64_t positions, int64_t heads) {
    return (batch == 1 || a[0] == b[0]) && (positions == 1 || a[1] == b[1]) && (heads == 1 || a[2] == b[2]);
}
// Whether an output that begins where an input does lies on it row by row: the same strides and, of keys and values, place i for token i
bool row_on_row(const lsp_rotary_problem* p, const void* in, const int64_t (&si)[3], const void* out, const int64_t (&so)[3], int64_t heads, bool placed) {
    return in != out || (same_strides(si, so, p->batch, p->length, heads) && (!placed || !p->starts));
}

int check_rotary(const lsp_rotary_problem* p, lsp_dtype t) {
    if (!p || !p->Q || !p->K || !p->Qr || !p->Kr || !p->V != !p->Vr || (p->rotated > 0 && !p->frequencies)) return LSP_ERR_NULL;
    int rc = check_rotary_shape(p, t);
    if (rc != LSP_OK) return rc;
    if (!(p->eps >= 0.0f) || !std::isfinite(p->eps)) return LSP_ERR_VALUE;
    if ((rc = check_heads(p->q_stride, p->batch, p->length, p->heads, p->head_dim, t, false)) != LSP_OK) return rc;
    if ((rc = check_heads(p->k_stride, p->batch, p->length, p->kv_heads, p->head_dim, t, false)) != LSP_OK) return rc;
    if ((rc = check_heads(p->qr_stride, p->batch, p->length, p->heads, p->head_dim, t, true)) != LSP_OK) return rc;
    if ((rc = check_heads(p->kr_stride, p->batch, p->cache, p->kv_heads, p->head_dim, t, true)) != LSP_OK) return rc;
    if (p->V) {
        if ((rc = check_heads(p->v_stride, p->batch, p->length, p->kv_heads, p->head_dim, t, false)) != LSP_OK) return rc;
        if ((rc = check_heads(p->vr_stride, p->batch, p->cache, p->kv_heads, p->head_dim, t, true)) != LSP_OK) return rc;
    }
    for (const void* q : {p->Q, p->K, p->V, static_cast<const void*>(p->Qr), static_cast<const void*>(p->Kr), static_cast<const void*>(p->Vr), p->q_weight, p->k_weight, p->q_bias, p->k_bias,
                          static_cast<const void*>(p->frequencies)})
        if (!aligned16(q)) return LSP_ERR_ALIGN;
    if ((reinterpret_cast<uintptr_t>(p->positions) | reinterpret_cast<uintptr_t>(p->starts) | reinterpret_cast<uintptr_t>(p->lens)) & 3u) return LSP_ERR_ALIGN;
    if (!row_on_row(p, p->Q, p->q_stride, p->Qr, p->qr_stride, p->heads, false) || !row_on_row(p, p->K, p->k_stride, p->Kr, p->kr_stride, p->kv_heads, true) ||
        (p->V && !row_on_row(p, p->V, p->v_stride, p->Vr, p->vr_stride, p->kv_heads, true)))
        return LSP_ERR_SHAPE;
    return LSP_OK;
}

lsp::RotaryArgs rotary_args(const lsp_rotary_problem* p) {
    lsp::RotaryArgs a{};
    auto &q = a.segment[0], &k = a.segment[1], &v = a.segment[2];
    q.x = strided(p->Q, p->q_stride, p->batch, p->length, p->heads);
    k.x = strided(p->K, p->k_stride, p->batch, p->length, p->kv_heads);
    q.y = strided(p->Qr, p->qr_stride, p->batch, p->length, p->heads);
    k.y = strided(p->Kr, p->kr_stride, p->batch, p->cache, p->kv_heads);
    if (p->V) {
        v.x = strided(p->V, p->v_stride, p->batch, p->length, p->kv_heads);
        v.y = strided(p->Vr, p->vr_stride, p->batch, p->cache, p->kv_heads);
    }
    q.heads = p->heads; k.heads = v.heads = p->kv_heads; k.placed = v.placed = 1;
    q.weight = p->q_weight; k.weight = p->k_weight; q.bias = p->q_bias; k.bias = p->k_bias;
    a.frequencies = p->frequencies; a.positions = p->positions; a.starts = p->starts; a.lens = p->lens;
    a.batch = p->batch; a.length = p->length; a.cache = p->cache; a.head_dim = p->head_dim;
    a.rotated = p->rotated; a.neighbours = p->neighbours; a.norm = p->norm; a.eps = p->eps;
    a.segments = p->V ? 3 : 2;
    return a;
}
lsp::RotaryArgs rotary_back_args(const lsp_rotary_problem* p, bool sums) {
    lsp::RotaryArgs a = rotary_args(p);
    a.segments = 2;
    a.sums = sums;
    lsp::plan_rotary(a, true);
    return a;
}

int check_loss_shape(const lsp_cross_entropy_problem* p, lsp_dtype t) {
    if (!p) return LSP_ERR_NULL;
    if (p->rows <= 0 || p->rows > LSP_MAX_ROWS || p->width <= 0 || p->width > (1 << 16) || p->width % 8 || p->vocab <= 0 || p->vocab > (1 << 20)) return LSP_ERR_SHAPE;
    if (!known(t)) return LSP_ERR_DTYPE;
    if (!(p->smoothing >= 0.0f && p->smoothing < 1.0f) || !(p->z_loss >= 0.0f && p->z_loss <= 1.0f)) return LSP_ERR_VALUE;
    return LSP_OK;
}
// A matrix's row stride: multiples of 16 bytes, below 8 MiB
int check_matrix(int64_t rows, int64_t width, int64_t stride, lsp_dtype t) {
    if (rows == 1) return LSP_OK;                                         // (not used)
    if (stride < width || stride * elem_size(t) >= (8 << 20)) return LSP_ERR_SHAPE;
    return stride * elem_size(t) % 16 ? LSP_ERR_ALIGN : LSP_OK;
}
int check_loss(const lsp_cross_entropy_problem* p, lsp_dtype t) {
    if (!p || !p->H || !p->W || !p->targets || !p->losses) return LSP_ERR_NULL;
    int rc = check_loss_shape(p, t);
    if (rc != LSP_OK) return rc;
    if ((rc = check_matrix(p->rows, p->width, p->h_stride, t)) != LSP_OK || (rc = check_matrix(p->vocab, p->width, p->w_stride, t)) != LSP_OK) return rc;
    for (const void* q : {p->H, p->W, static_cast<const void*>(p->targets), static_cast<const void*>(p->losses), static_cast<const void*>(p->logs)})
        if (!aligned16(q)) return LSP_ERR_ALIGN;
    return LSP_OK;
}
lsp::LossArgs loss_args(const lsp_cross_entropy_problem* p, bool train, lsp_dtype t) {
    lsp::LossArgs a{};
    a.H = p->H; a.W = p->W; a.targets = p->targets; a.losses = p->losses; a.logs = p->logs;
    a.h_stride = p->rows > 1 ? p->h_stride : p->width; a.w_stride = p->vocab > 1 ? p->w_stride : p->width;
    a.rows = p->rows; a.width = p->width; a.vocab = p->vocab; a.smoothing = p->smoothing; a.z_loss = p->z_loss;
    a.train = train;
    lsp::plan_loss(a, t);
    return a;
}

template <bool BITS8> int adamw_launches(const lsp_adamw_item* items, int32_t count, double rate, double beta1, double beta2, double eps, int64_t step, const float* grad_scale, void* stream) {
    using Group = lsp::AdamwGroup<BITS8>;
    Group g{};
    const double c1 = 1.0 - std::pow(beta1, (double)step), root2 = std::sqrt(1.0 - std::pow(beta2, (double)step));
    // (sqrt(v) is 0 or at least 2^-75: FLT_MIN beside it changes nothing, and makes 0 / 0 of an element without any gradients so far 0)
    g.step = {(float)(1.0 - beta1), (float)beta1, (float)(1.0 - beta2), (float)beta2, std::max((float)(eps * root2), FLT_MIN), (float)(rate * root2 / c1), (float)rate};
    g.one_minus_beta1 = 1.0 - beta1; g.beta1 = beta1; g.one_minus_beta2 = 1.0 - beta2; g.beta2 = beta2;
    g.grad_scale = grad_scale;
    for (int32_t first = 0; first < count; first += Group::kItems) {
        uint32_t total = 0;
        for (int k = 0; k < Group::kItems; ++k) {
            g.first[k] = first + k < count ? (int32_t)total : INT32_MAX;
            if (first + k >= count) continue;
            const lsp_adamw_item& i = items[first + k];
            auto& to = g.item[k];
            to.param = i.param; to.grad = i.grad; to.m = i.m; to.v = i.v; to.master = i.master;
            to.elements = (i.dtype + 4 * i.grad_dtype) * lsp::kAdamwSizes + i.elements;
            to.rate_factor = i.rate_factor; to.decay = i.decay;
            if constexpr (BITS8) { to.m_scale = i.m_scale; to.v_scale = i.v_scale; }
            total += (uint32_t)((i.elements + lsp::kAdamwElements - 1) / lsp::kAdamwElements);
        }
        const int rc = done(lsp::launch_adamw<BITS8>(g, total, static_cast<hipStream_t>(stream)));
        if (rc != LSP_OK) return rc;
    }
    return LSP_OK;
}

}  // namespace

extern "C" {

int lsp_rotary_forward(const lsp_rotary_problem* p, lsp_dtype dtype, void* stream) {
    const int rc = check_rotary(p, dtype);
    if (rc != LSP_OK) return rc;
    lsp::RotaryArgs a = rotary_args(p);
    lsp::plan_rotary(a, false);
    if (a.blocks >= kMostLaunch) return LSP_ERR_SHAPE;
    return done(lsp::launch_rotary(a, false, dtype, static_cast<hipStream_t>(stream)));
}

size_t lsp_rotary_backward_workspace_bytes(const lsp_rotary_problem* p, lsp_dtype dtype) {
    if (check_rotary_shape(p, dtype) != LSP_OK) return 0;
    return p->norm == LSP_NORM_NONE ? 0 : lsp::rotary_partial_bytes(rotary_back_args(p, true));
}

int lsp_rotary_backward(const lsp_rotary_problem* p, const lsp_rotary_gradients* g, lsp_dtype dtype, void* workspace, size_t workspace_bytes, void* stream) {
    if (!p || !g || !g->dQr || !g->dKr || !g->dQ || !g->dK) return LSP_ERR_NULL;
    int rc = check_rotary(p, dtype);
    if (rc != LSP_OK) return rc;
    if ((rc = check_heads(g->dqr_stride, p->batch, p->length, p->heads, p->head_dim, dtype, false)) != LSP_OK) return rc;
    if ((rc = check_heads(g->dkr_stride, p->batch, p->cache, p->kv_heads, p->head_dim, dtype, false)) != LSP_OK) return rc;
    if ((rc = check_heads(g->dq_stride, p->batch, p->length, p->heads, p->head_dim, dtype, true)) != LSP_OK) return rc;
    if ((rc = check_heads(g->dk_stride, p->batch, p->length, p->kv_heads, p->head_dim, dtype, true)) != LSP_OK) return rc;
    for (const void* q : {g->dQr, g->dKr, static_cast<const void*>(g->dQ), static_cast<const void*>(g->dK), static_cast<const void*>(g->q_weight), static_cast<const void*>(g->k_weight),
                          static_cast<const void*>(g->q_bias), static_cast<const void*>(g->k_bias)})
        if (!aligned16(q)) return LSP_ERR_ALIGN;
    if (!row_on_row(p, g->dQr, g->dqr_stride, g->dQ, g->dq_stride, p->heads, false) || !row_on_row(p, p->Q, p->q_stride, g->dQ, g->dq_stride, p->heads, false) ||
        !row_on_row(p, g->dKr, g->dkr_stride, g->dK, g->dk_stride, p->kv_heads, true) || !row_on_row(p, p->K, p->k_stride, g->dK, g->dk_stride, p->kv_heads, false))
        return LSP_ERR_SHAPE;
    const bool normed = p->norm != LSP_NORM_NONE;
    if (normed && (p->Qr == p->Q || p->Kr == p->K)) return LSP_ERR_SHAPE;                // what was normed is needed as it was
    const bool sums = g->q_weight || g->k_weight || g->q_bias || g->k_bias;
    if (sums && !normed) return LSP_ERR_SHAPE;                                           // a norm that is none has no weights
    lsp::RotaryArgs a = rotary_back_args(p, sums);
    if (a.blocks >= kMostLaunch) return LSP_ERR_SHAPE;
    const size_t need = lsp::rotary_partial_bytes(a);
    if (need && (!workspace || workspace_bytes < need || !aligned16(workspace))) return LSP_ERR_WORKSPACE;
    a.partial = static_cast<float*>(workspace);
    auto &q = a.segment[0], &k = a.segment[1];
    q.y = strided(g->dQr, g->dqr_stride, p->batch, p->length, p->heads);
    k.y = strided(g->dKr, g->dkr_stride, p->batch, p->cache, p->kv_heads);
    q.out = strided(g->dQ, g->dq_stride, p->batch, p->length, p->heads);
    k.out = strided(g->dK, g->dk_stride, p->batch, p->length, p->kv_heads);
    q.weight_sum = g->q_weight; k.weight_sum = g->k_weight; q.bias_sum = g->q_bias; k.bias_sum = g->k_bias;
    return done(lsp::launch_rotary(a, true, dtype, static_cast<hipStream_t>(stream)));
}

size_t lsp_cross_entropy_forward_workspace_bytes(const lsp_cross_entropy_problem* p, lsp_dtype dtype) {
    if (check_loss_shape(p, dtype) != LSP_OK) return 0;
    lsp::LossArgs a = loss_args(p, false, dtype);
    return lsp::loss_workspace(a, dtype, nullptr);
}

int lsp_cross_entropy_forward(const lsp_cross_entropy_problem* p, lsp_dtype dtype, void* workspace, size_t workspace_bytes, void* stream) {
    const int rc = check_loss(p, dtype);
    if (rc != LSP_OK) return rc;
    lsp::LossArgs a = loss_args(p, false, dtype);
    if (!workspace || !aligned16(workspace) || workspace_bytes < lsp::loss_workspace(a, dtype, nullptr)) return LSP_ERR_WORKSPACE;
    lsp::loss_workspace(a, dtype, static_cast<uint8_t*>(workspace));
    return done(lsp::launch_loss(a, dtype, static_cast<hipStream_t>(stream)));
}

size_t lsp_cross_entropy_backward_workspace_bytes(const lsp_cross_entropy_problem* p, lsp_dtype dtype) {
    if (check_loss_shape(p, dtype) != LSP_OK) return 0;
    lsp::LossArgs a = loss_args(p, true, dtype);
    return lsp::loss_workspace(a, dtype, nullptr);
}

int lsp_cross_entropy_backward(const lsp_cross_entropy_problem* p, const lsp_cross_entropy_gradients* g, lsp_dtype dtype, void* workspace, size_t workspace_bytes, void* stream) {
    if (!p || !g || (!g->dH && !g->dW)) return LSP_ERR_NULL;
    int rc = check_loss(p, dtype);
    if (rc != LSP_OK) return rc;
    if (!std::isfinite(g->scale)) return LSP_ERR_VALUE;
    if (g->dH && (rc = check_matrix(p->rows, p->width, g->dh_stride, dtype)) != LSP_OK) return rc;
    if (g->dW && (rc = check_matrix(p->vocab, p->width, g->dw_stride, dtype)) != LSP_OK) return rc;
    if (!aligned16(g->dH) || !aligned16(g->dW) || !aligned16(g->weights)) return LSP_ERR_ALIGN;
    if (g->dH == p->H || g->dW == p->W || g->dH == p->W || g->dW == p->H) return LSP_ERR_SHAPE;      // both are needed as they are until the last kernel
    lsp::LossArgs a = loss_args(p, true, dtype);
    if (!workspace || !aligned16(workspace) || workspace_bytes < lsp::loss_workspace(a, dtype, nullptr)) return LSP_ERR_WORKSPACE;
    lsp::loss_workspace(a, dtype, static_cast<uint8_t*>(workspace));
    a.dH = g->dH; a.dW = g->dW; a.weights = g->weights; a.scale = g->scale;
    a.dh_stride = p->rows > 1 ? g->dh_stride : p->width; a.dw_stride = p->vocab > 1 ? g->dw_stride : p->width;
    return done(lsp::launch_loss(a, dtype, static_cast<hipStream_t>(stream)));
}

int lsp_adamw(const lsp_adamw_item* items, int32_t count, lsp_state states, double rate, double beta1, double beta2, double eps, int64_t step,
              const float* grad_scale, void* stream) {
    if (!items) return LSP_ERR_NULL;
    if (count <= 0 || count > LSP_MAX_TENSORS || step < 1 || (states != LSP_STATE_F32 && states != LSP_STATE_8BIT)) return LSP_ERR_SHAPE;
    if (!std::isfinite(rate) || !(beta1 >= 0.0 && beta1 < 1.0) || !(beta2 >= 0.0 && beta2 < 1.0) || !(eps >= 0.0) || !std::isfinite(eps)) return LSP_ERR_VALUE;
    if (reinterpret_cast<uintptr_t>(grad_scale) & 3u) return LSP_ERR_ALIGN;
    const bool bits8 = states == LSP_STATE_8BIT;
    int64_t blocks = 0;
    for (int32_t k = 0; k < count; ++k) {
        const lsp_adamw_item& i = items[k];
        if (!i.param || !i.grad || !i.m || !i.v || (bits8 && (!i.m_scale || !i.v_scale))) return LSP_ERR_NULL;
        if (i.elements <= 0 || i.elements > (int64_t)1 << 35) return LSP_ERR_SHAPE;
        if (!known(static_cast<lsp_dtype>(i.dtype)) || !known(static_cast<lsp_dtype>(i.grad_dtype))) return LSP_ERR_DTYPE;
        if (!std::isfinite(i.rate_factor) || !std::isfinite(i.decay)) return LSP_ERR_VALUE;
        for (const void* q : {static_cast<const void*>(i.param), i.grad, static_cast<const void*>(i.m), static_cast<const void*>(i.v), static_cast<const void*>(i.master)})
            if (!aligned16(q)) return LSP_ERR_ALIGN;
        if (bits8 && ((reinterpret_cast<uintptr_t>(i.m_scale) | reinterpret_cast<uintptr_t>(i.v_scale)) & 3u)) return LSP_ERR_ALIGN;
        blocks += (i.elements + lsp::kAdamwElements - 1) / lsp::kAdamwElements;
        if (blocks >= kMostLaunch) return LSP_ERR_SHAPE;
    }
    return bits8 ? adamw_launches<true>(items, count, rate, beta1, beta2, eps, step, grad_scale, stream) : adamw_launches<false>(items, count, rate, beta1, beta2, eps, step, grad_scale, stream);
}

}  // extern "C"

// Norm after a block, gated residual with dropout, norm before the next block, in one pass over the rows; and its backward pass.
//
// Forward, for each row:  u = norm(f),  y = a x + b g drop(u),  h = norm(y).  A row stays in registers from its one load on (TPR
// threads, NV units of eight columns each); mean and deviation are two sums over the row each, the second of squares of what the mean
// leaves (so that a large mean costs no digits).
//
// Backward, with the gradients dy, dh that arrive and f^ = (f - mean) / deviation, y^ likewise:
//     e   = dh w_pre,            dY = dy + (e - mean(e) - y^ mean(e y^)) / deviation(y)        (RMS: without mean(e))
//     dx  = a dY,                du = keep b g dY
//     e'  = du w_post,           df = (e' - mean(e') - f^ mean(e' f^)) / deviation(f)
// and the sums over rows  dw_pre = dh y^, db_pre = dh, dg = b dY drop(u), dw_post = du f^, db_post = du.  y is made again from x and
// f, in fp32: nothing of the row is stored but its four statistics.  A workgroup goes through many rows and keeps its part of the sums over
// rows in registers; the parts are added by a second kernel in a fixed order, so the results do not depend on timing.
//
// Both are bound by memory, and nearly as much by the vector units: forward reads x and f and writes y and h (4096 x 4096, bf16, 134 MB: 23.6 us, 5.7 TB/s), backward reads x, f,
// dy, dh and writes dx, df (201 MB: 39 us, 5.1 TB/s), each once.
#include "residual_norm.h"
#include "rows.h"

namespace lsp {

constexpr int kGrads = 5;
typedef float f32x4 __attribute__((ext_vector_type(4)));

// Sums of N values over the TPR threads of a row, in all of them.  `scratch`: this row group's, two sets that take turns.
template <int TPR, int N> struct RowSum {
    float* scratch;                                       // LDS: [2][TPR / 64][N]
    int turn = 0;
    __device__ __forceinline__ void operator()(float (&v)[N]) {
#pragma unroll
        for (int k = 0; k < N; ++k) v[k] = wave_sum(v[k]);
        if constexpr (TPR > 64) {
            constexpr int kWaves = TPR / 64;
            const int lane = threadIdx.x & 63, wave = (threadIdx.x % TPR) >> 6;
            float* mine = scratch + turn * (kWaves * N);
            turn ^= 1;
            if (lane == 0)
#pragma unroll
                for (int k = 0; k < N; ++k) mine[wave * N + k] = v[k];
            __syncthreads();
#pragma unroll
            for (int k = 0; k < N; ++k) {
                float t = 0.0f;
#pragma unroll
                for (int w = 0; w < kWaves; ++w) t += mine[w * N + k];
                v[k] = t;
            }
        }
    }
};

// Columns of a thread: eight from `col` on.  The last thread of a row has the row's last eight, of which the first `others` are the thread's before it (and all eight, where the
// row has ended): they count in no sum and are not stored.  A block put together from smaller loads would wait for them at once, and every thread of the row for it (backward,
// 3001 rows: 2999 columns took 8 us longer than 3000, so 3).
struct Columns { int col, others; };
__device__ __forceinline__ Columns columns_of(int unit, int width) {
    const int col = min(unit * 8, width - 8);
    return {col, min(unit * 8 - col, 8)};
}

// Which of a thread's eight elements are kept, as bits
__device__ __forceinline__ uint32_t kept_bits(int64_t row, int unit, int others, int width, const Dropout& drop) {
    const uint64_t n = (uint64_t)row * (uint64_t)((width + 7) >> 3) + (uint64_t)unit;
    const u32x4 w = philox((uint32_t)n, (uint32_t)(n >> 32), 0, drop.offset, drop.key0, drop.key1);
    uint32_t bits = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) bits |= (philox_word(w, e) >= drop.limit ? 1u : 0u) << e;
    return bits << others;                                                                // (the block's words belong to the last columns)
}

// mean and 1 / deviation of a row, by kind; v becomes (v - mean) / deviation.  (Others' columns are set apart by branches that waves without such skip, not by selects for every element.)
template <int TPR, int NV> __device__ __forceinline__ void normalise(Eight (&v)[NV], const Columns (&c)[NV], int kind, int width, float eps, RowSum<TPR, 1>& sum, float& mean, float& rstd) {
    mean = 0.0f; rstd = 1.0f;
    if (kind == LSP_NORM_NONE) return;
    const float per = 1.0f / (float)width;
    const auto others_are_zero = [&] {
#pragma unroll
        for (int n = 0; n < NV; ++n)
            if (c[n].others)
#pragma unroll
                for (int e = 0; e < 8; ++e) v[n].x[e] = e >= c[n].others ? v[n].x[e] : 0.0f;
    };
    others_are_zero();
    if (kind == LSP_NORM_LAYER) {
        float s[1] = {0.0f};
#pragma unroll
        for (int n = 0; n < NV; ++n)
#pragma unroll
            for (int e = 0; e < 8; ++e) s[0] += v[n].x[e];
        sum(s);
        mean = s[0] * per;
#pragma unroll
        for (int n = 0; n < NV; ++n)
#pragma unroll
            for (int e = 0; e < 8; ++e) v[n].x[e] -= mean;
        others_are_zero();
    }
    float s[1] = {0.0f};
#pragma unroll
    for (int n = 0; n < NV; ++n)
#pragma unroll
        for (int e = 0; e < 8; ++e) s[0] = fmaf(v[n].x[e], v[n].x[e], s[0]);
    sum(s);
    rstd = 1.0f / sqrtf(s[0] * per + eps);
#pragma unroll
    for (int n = 0; n < NV; ++n)
#pragma unroll
        for (int e = 0; e < 8; ++e) v[n].x[e] *= rstd;
}

// v := v w + b, with ones and zeros where these are not there
template <typename D> __device__ __forceinline__ void weigh(Eight& v, const Packed<D>& w, const Packed<D>& b, bool weight, bool bias) {
    if (weight)
#pragma unroll
        for (int e = 0; e < 8; ++e) v.x[e] *= element<D>(w, e);
    if (bias)
#pragma unroll
        for (int e = 0; e < 8; ++e) v.x[e] += element<D>(b, e);
}

// A weight's or bias' columns, if it has some
template <typename D> __device__ __forceinline__ void ask_for(Packed<D>& v, const void* p, const Columns& c, bool whole) {
    if (p) v = load_ending<D>(static_cast<const typename D::elem*>(p) + c.col, c.others, whole);
}

template <typename D, int TPR, int NV, int GROUPS, bool DROP>
__global__ __launch_bounds__(TPR * GROUPS) void k_residual_norm(const ResidualNormArgs a) {
    using elem = typename D::elem;
    __shared__ float scratch[GROUPS][2 * (TPR / 64)];
    const int group = threadIdx.x / TPR, t = threadIdx.x % TPR;
    const int64_t row_asked = (int64_t)blockIdx.x * GROUPS + group;
    const int64_t row = row_asked < a.rows ? row_asked : a.rows - 1;                      // (every thread goes to every barrier)
    const bool mine = row_asked < a.rows;
    const int width = a.width;
    RowSum<TPR, 1> sum{scratch[group]};
    const elem* x = static_cast<const elem*>(a.x) + row * a.x_stride;
    const elem* f = static_cast<const elem*>(a.f) + row * a.f_stride;
    const bool whole = a.whole, x_whole = a.whole_too;
    Columns c[NV];
    Eight xv[NV], fv[NV];
#pragma unroll
    for (int n = 0; n < NV; ++n) {
        c[n] = columns_of(t + n * TPR, width);
        xv[n] = widen_eight<D>(load_ending<D>(x + c[n].col, c[n].others, x_whole));
        fv[n] = widen_eight<D>(load_ending<D>(f + c[n].col, c[n].others, whole));
    }
    // What the row is multiplied with is asked for before the sums that come first (4096 x 4096, layer norms with biases and dropout, fp16: 31 to 26 us).
    const bool post = a.post != LSP_NORM_NONE, pre = a.pre != LSP_NORM_NONE;
    const void *post_w = post ? a.post_w : nullptr, *post_b = post ? a.post_b : nullptr, *pre_w = pre ? a.pre_w : nullptr, *pre_b = pre ? a.pre_b : nullptr;
    Packed<D> w[NV], b[NV], g[NV];
#pragma unroll
    for (int n = 0; n < NV; ++n) { ask_for<D>(w[n], post_w, c[n], whole); ask_for<D>(b[n], post_b, c[n], whole); ask_for<D>(g[n], a.gate, c[n], whole); }
    float mean_f, rstd_f, mean_y, rstd_y;
    normalise<TPR, NV>(fv, c, a.post, width, a.eps, sum, mean_f, rstd_f);
#pragma unroll
    for (int n = 0; n < NV; ++n) {
        weigh<D>(fv[n], w[n], b[n], post_w, post_b);
        float scale = a.branch_scale;
        if constexpr (DROP) {
            const uint32_t kept = kept_bits(row, t + n * TPR, c[n].others, width, a.drop);
#pragma unroll
            for (int e = 0; e < 8; ++e) fv[n].x[e] = kept >> e & 1u ? fv[n].x[e] : 0.0f;
            scale *= a.drop.scale;
        }
        if (a.gate)
#pragma unroll
            for (int e = 0; e < 8; ++e) fv[n].x[e] *= element<D>(g[n], e);
#pragma unroll
        for (int e = 0; e < 8; ++e) xv[n].x[e] = fmaf(scale, fv[n].x[e], a.residual_scale * xv[n].x[e]);
        if (mine) store_ending<D>(static_cast<elem*>(a.y) + row * a.y_stride + c[n].col, xv[n], c[n].others);
        ask_for<D>(w[n], pre_w, c[n], whole);
        ask_for<D>(b[n], pre_b, c[n], whole);
    }
    normalise<TPR, NV>(xv, c, a.pre, width, a.eps, sum, mean_y, rstd_y);
    if (mine && a.h) {
#pragma unroll
        for (int n = 0; n < NV; ++n) {
            weigh<D>(xv[n], w[n], b[n], pre_w, pre_b);
            store_ending<D>(static_cast<elem*>(a.h) + row * a.h_stride + c[n].col, xv[n], c[n].others);
        }
    }
    if (mine && t == 0) {
        a.stats[row] = mean_f; a.stats[a.rows + row] = rstd_f;
        a.stats[2 * a.rows + row] = mean_y; a.stats[3 * a.rows + row] = rstd_y;
    }
}

// A thread has NV units of eight columns, TPR threads a row and GROUPS rows a workgroup.  With one workgroup a CU, what is on the way is what its rows ask for, so the rows of the
// next two steps are (one step ahead, 16384 x 2048 took 115 us, with two 90; wide rows, NV = 2, have registers for one).  Beside memory the instructions count, some 60 an
// element: weights stay in registers, in fp32, and what can be folded into a factor of the row is (4096 x 4096: 47 to 42 us, 3001 x 3000 with biases 49 to 37).
// BIAS: a norm has a bias, or the gradient of one is asked for.
template <typename D, int TPR, int NV, int GROUPS, bool DROP, bool BIAS>
__global__ __launch_bounds__(TPR * GROUPS, 2) void k_residual_norm_back(const ResidualNormArgs a) {
    using elem = typename D::elem;
    constexpr int kSumFloats = GROUPS * 4 * (TPR / 64), AHEAD = NV == 1 ? 2 : 1;
    __shared__ float scratch[GROUPS > 1 ? (GROUPS - 1) * TPR * 8 : kSumFloats];           // RowSum's, and at the end the other groups' sums over rows
    const int group = __builtin_amdgcn_readfirstlane(threadIdx.x / TPR), t = threadIdx.x % TPR;
    const int width = a.width;
    Columns c[NV];
#pragma unroll
    for (int n = 0; n < NV; ++n) c[n] = columns_of(t + n * TPR, width);
    const bool whole = a.whole, dy_whole = a.whole_too;
    const float per = 1.0f / (float)width, scale_u = DROP ? a.branch_scale * a.drop.scale : a.branch_scale;
    RowSum<TPR, 2> sum{scratch + group * 4 * (TPR / 64)};
    const bool post = a.post != LSP_NORM_NONE, pre = a.pre != LSP_NORM_NONE;
    // Weights stay in registers, in fp32, while these have room (NV = 1), else in LDS as they came, where each thread reads what it wrote, a unit at a time; as packed registers
    // they made others spill (4096 x 8192, fp32: 253 us, so 165).
    constexpr bool HELD = NV == 1;
    constexpr int kPieces = D::size / 2;                                                  // of 16 bytes, of eight elements
    enum { WF, G, BF, WY };
    constexpr int kInLds = BIAS && D::size == 4 ? 2 : 4;                                  // (LDS has not room for all; the others are read again, from the caches)
    __shared__ u32x4 kept_weights[HELD ? 1 : kInLds * NV * kPieces * TPR];
    float held[HELD ? 4 : 1][8];
    const auto vector = [&](int which, int n) {
        const void* p = which == WF ? (post ? a.post_w : nullptr) : which == BF ? (post ? a.post_b : nullptr) : which == G ? a.gate : pre ? a.pre_w : nullptr;
        const float otherwise = which == BF ? 0.0f : 1.0f;
        const int first = which == G || which == WY ? c[n].others : 0;                    // (zeros for others' columns: they add nothing to any sum)
        Eight r;
        if (p) r = widen_eight<D>(load_ending<D>(static_cast<const elem*>(p) + c[n].col, c[n].others, whole));
#pragma unroll
        for (int e = 0; e < 8; ++e) r.x[e] = e < first ? 0.0f : p ? r.x[e] : otherwise;
        return r;
    };
#pragma unroll
    for (int n = 0; n < NV; ++n)
#pragma unroll
        for (int which = 0; which < (HELD ? 4 : kInLds); ++which) {
            if (which == BF && !BIAS) continue;
            const Eight r = vector(which, n);
            if constexpr (HELD) {
#pragma unroll
                for (int e = 0; e < 8; ++e) held[which][e] = r.x[e];
            } else {
                const Packed<D> v = narrow_eight<D>(r);
#pragma unroll
                for (int k = 0; k < kPieces; ++k) kept_weights[((which * NV + n) * kPieces + k) * TPR + t] = u32x4{v.w[4 * k], v.w[4 * k + 1], v.w[4 * k + 2], v.w[4 * k + 3]};
            }
        }
    struct Weights { Packed<D> v[HELD ? 1 : 4]; };
    const auto weights_of = [&](Weights& w, int n, bool all) {                            // for the next eight columns
        if constexpr (!HELD)
#pragma unroll
            for (int which = 0; which < 4; ++which) {
                if ((which == BF && !BIAS) || (which == WY && !all)) continue;
                if (which >= kInLds) { w.v[which] = narrow_eight<D>(vector(which, n)); continue; }
#pragma unroll
                for (int k = 0; k < kPieces; ++k) {
                    const u32x4 v = kept_weights[((which * NV + n) * kPieces + k) * TPR + t];
#pragma unroll
                    for (int i = 0; i < 4; ++i) w.v[which].w[4 * k + i] = v[i];
                }
            }
    };
    const auto of = [&](const Weights& w, int which, int e) { if constexpr (HELD) return held[which][e]; else return element<D>(w.v[which], e); };
    float acc[NV][kGrads][8];
#pragma unroll
    for (int n = 0; n < NV; ++n)
#pragma unroll
        for (int k = 0; k < kGrads; ++k)
#pragma unroll
            for (int e = 0; e < 8; ++e) acc[n][k][e] = 0.0f;
    // The biases' sums of wide rows are in LDS too, where each thread adds to its own (4096 x 8192, layer norms with dropout: fp16 98 us, in registers, which spill, 196; fp32 286 and 509).
    constexpr bool SUMS_IN_LDS = BIAS && !HELD;
    __shared__ f32x4 bias_sums[SUMS_IN_LDS ? 2 * NV * 2 * TPR : 1];
    const auto bias_sum = [&](int which, int n, int half) -> f32x4& { return bias_sums[((which * NV + n) * 2 + half) * TPR + t]; };
    if constexpr (SUMS_IN_LDS)
#pragma unroll
        for (int k = 0; k < 4 * NV; ++k) bias_sums[k * TPR + t] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    const auto add_to_bias = [&](int which, int n, const float (&v)[8]) {
#pragma unroll
        for (int half = 0; half < 2; ++half) bias_sum(which, n, half) += f32x4{v[4 * half], v[4 * half + 1], v[4 * half + 2], v[4 * half + 3]};
    };
    // What belongs to a row is asked for AHEAD rows before.
    struct Row { Packed<D> x[NV], f[NV], dy[NV], dh[NV]; float stats[4]; };
    Row rows_[AHEAD];
    uint32_t lane0 = 0;                                                                   // (statistics come into vector registers, as the rest does: a scalar load would be waited for with LDS)
    asm volatile("" : "+v"(lane0));
    // A group without a row (every thread goes to every barrier) has the last row with gradients of zeros: it adds zeros, and stores nothing.
    const auto load_first = [&](Row& r, int64_t base) {
        const int64_t row = base + group < a.rows ? base + group : a.rows - 1;
        const elem* x = static_cast<const elem*>(a.x) + row * a.x_stride;
        const elem* f = static_cast<const elem*>(a.f) + row * a.f_stride;
        const elem* dh = a.dh ? static_cast<const elem*>(a.dh) + row * a.dh_stride : x;
#pragma unroll
        for (int k = 0; k < 4; ++k) r.stats[k] = (a.stats + k * a.rows + row)[lane0];
#pragma unroll
        for (int n = 0; n < NV; ++n) {
            const int col = c[n].col, first = base + group < a.rows ? c[n].others : 8;     // (zeros where the group has no row: its sums then get zeros)
            r.x[n] = load_ending<D>(x + col, first, whole);
            r.f[n] = load_ending<D>(f + col, first, whole);
            r.dh[n] = load_ending<D>(dh + col, a.dh ? first : 8, whole);
        }
    };
    const auto load_dy = [&](Row& r, int64_t base) {
        const int64_t row = base + group < a.rows ? base + group : a.rows - 1;
#pragma unroll
        for (int n = 0; n < NV; ++n) r.dy[n] = load_ending<D>(static_cast<const elem*>(a.dy) + row * a.dy_stride + c[n].col, base + group < a.rows ? c[n].others : 8, dy_whole);
    };
    const int64_t step = (int64_t)gridDim.x * GROUPS, first = (int64_t)blockIdx.x * GROUPS;
    const auto one_row = [&](Row& r, int64_t base) {
        const bool mine = GROUPS == 1 || base + group < a.rows;
        const int64_t row = base + group < a.rows ? base + group : a.rows - 1, next = base + AHEAD * step;
        const float mean_f = r.stats[0], rstd_f = r.stats[1], mean_y = r.stats[2], rstd_y = r.stats[3];
        // y^ and f^, and the gradient of y^
        uint32_t kept[NV];
        float fhat[NV][8], yhat[NV][8], de[NV][8], s[2] = {0.0f, 0.0f};
#pragma unroll
        for (int n = 0; n < NV; ++n) {
            if constexpr (DROP) kept[n] = kept_bits(row, t + n * TPR, c[n].others, width, a.drop);
            Weights w;
            weights_of(w, n, true);
            float to_bias[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                if (e % 4 == 0) __builtin_amdgcn_sched_barrier(0);                        // (four at a time: eight would take registers for speed that nothing waits for)
                const float wf = of(w, WF, e), bf = BIAS ? of(w, BF, e) : 0.0f, gate = of(w, G, e), wy = of(w, WY, e);
                fhat[n][e] = (element<D>(r.f[n], e) - mean_f) * rstd_f;
                const float u = !DROP ? fmaf(fhat[n][e], wf, bf) : (kept[n] >> e & 1u) ? fmaf(fhat[n][e], wf, bf) : 0.0f;   // (what is dropped may be infinite)
                yhat[n][e] = fmaf(scale_u * gate, u, fmaf(a.residual_scale, element<D>(r.x[n], e), -mean_y)) * rstd_y;
                const float d = element<D>(r.dh[n], e);
                acc[n][0][e] = fmaf(d, yhat[n][e], acc[n][0][e]);
                if constexpr (SUMS_IN_LDS) to_bias[e] = d;
                else if constexpr (BIAS) acc[n][1][e] += d;
                de[n][e] = d * wy;
                s[0] = fmaf(de[n][e], yhat[n][e], s[0]);
                s[1] += de[n][e];
            }
            if constexpr (SUMS_IN_LDS) add_to_bias(0, n, to_bias);
        }
        load_first(r, next);                                                              // (where what they held is used up)
        if (pre) sum(s);
        float s1 = pre ? s[0] * per * rstd_y : 0.0f, s0 = a.pre == LSP_NORM_LAYER ? s[1] * per * rstd_y : 0.0f;
        s[0] = s[1] = 0.0f;
#pragma unroll
        for (int n = 0; n < NV; ++n) {
            Eight out;
            Weights w;
            weights_of(w, n, false);
            float to_bias[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                if (e % 4 == 0) __builtin_amdgcn_sched_barrier(0);
                const float wf = of(w, WF, e), bf = BIAS ? of(w, BF, e) : 0.0f, gate = of(w, G, e);
                const float dy = element<D>(r.dy[n], e), total = pre ? fmaf(de[n][e], rstd_y, dy - s0) - yhat[n][e] * s1 : dy + de[n][e];
                out.x[e] = a.residual_scale * total;
                const float branch = !DROP || (kept[n] >> e & 1u) ? total : 0.0f, u = !DROP || (kept[n] >> e & 1u) ? fmaf(fhat[n][e], wf, bf) : 0.0f;
                const float du = branch * (scale_u * gate);
                acc[n][2][e] = fmaf(branch, u, acc[n][2][e]);
                acc[n][3][e] = fmaf(du, fhat[n][e], acc[n][3][e]);
                if constexpr (SUMS_IN_LDS) to_bias[e] = du;
                else if constexpr (BIAS) acc[n][4][e] += du;
                de[n][e] = du * wf;
                s[0] = fmaf(de[n][e], fhat[n][e], s[0]);
                s[1] += de[n][e];
            }
            if constexpr (SUMS_IN_LDS) add_to_bias(1, n, to_bias);
            if (mine) store_ending<D>(static_cast<elem*>(a.dx) + row * a.dx_stride + c[n].col, out, c[n].others);
        }
        load_dy(r, next);
        if (post) sum(s);
        s1 = s[0] * per * rstd_f; s0 = a.post == LSP_NORM_LAYER ? s[1] * per * rstd_f : 0.0f;
#pragma unroll
        for (int n = 0; n < NV; ++n) {
            Eight out;
#pragma unroll
            for (int e = 0; e < 8; ++e) out.x[e] = post ? fmaf(de[n][e], rstd_f, -s0) - fhat[n][e] * s1 : de[n][e];
            if (mine) store_ending<D>(static_cast<elem*>(a.df) + row * a.df_stride + c[n].col, out, c[n].others);
        }
    };
#pragma unroll
    for (int k = 0; k < AHEAD; ++k) { load_first(rows_[k], first + k * step); load_dy(rows_[k], first + k * step); }
    for (int64_t base = first; base < a.rows; base += AHEAD * step) {
        one_row(rows_[0], base);
        if constexpr (AHEAD > 1)
            if (base + step < a.rows) one_row(rows_[1], base + step);
    }
    // the workgroup's part of the sums over rows
    int slot = 0;
#pragma unroll
    for (int k = 0; k < kGrads; ++k) {
        if (!a.grads[k]) continue;
#pragma unroll
        for (int n = 0; n < NV; ++n) {
            Eight v;
#pragma unroll
            for (int e = 0; e < 8; ++e) v.x[e] = (SUMS_IN_LDS && (k == 1 || k == 4) ? bias_sum(k == 4, n, e >> 2)[e & 3] : acc[n][k][e]) * (k == 2 ? scale_u : 1.0f);
            if (GROUPS > 1 && !a.many) {                                                  // (few rows: every group's part by itself, the adding is short)
                store_ending<F32>(a.partial + (((int64_t)slot * gridDim.x + blockIdx.x) * GROUPS + group) * width + c[n].col, v, c[n].others);
                continue;
            }
            if constexpr (GROUPS > 1) {
                __syncthreads();                                                          // (scratch is free)
                if (group > 0)
#pragma unroll
                    for (int e = 0; e < 8; ++e) scratch[((group - 1) * 8 + e) * TPR + t] = v.x[e];
                __syncthreads();
                if (group == 0)
#pragma unroll
                    for (int o = 0; o < GROUPS - 1; ++o)
#pragma unroll
                        for (int e = 0; e < 8; ++e) v.x[e] += scratch[(o * 8 + e) * TPR + t];
            }
            if (group == 0) store_ending<F32>(a.partial + ((int64_t)slot * gridDim.x + blockIdx.x) * width + c[n].col, v, c[n].others);
        }
        ++slot;
    }
}

// Adds the parts: a workgroup has 32 columns of one sum, its 32 rows of threads take turns at the parts.
__global__ __launch_bounds__(1024) void k_residual_norm_sums(const ResidualNormArgs a, int parts) {
    __shared__ float add[32][33];
    const int x = threadIdx.x & 31, y = threadIdx.x >> 5;
    const int col = blockIdx.x * 32 + x;
    float* out = nullptr;
    int slot = 0;
#pragma unroll
    for (int k = 0; k < kGrads; ++k)
        if (a.grads[k]) { if (slot == (int)blockIdx.y) out = a.grads[k]; ++slot; }
    const float* p = a.partial + (int64_t)blockIdx.y * parts * a.width;
    float s = 0.0f;
    if (col < a.width)
#pragma unroll 1
        for (int r = y; r < parts; r += 32 * 8) {                                         // (eight on the way at a time)
            float v[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) v[k] = r + 32 * k < parts ? p[(int64_t)(r + 32 * k) * a.width + col] : 0.0f;
#pragma unroll
            for (int k = 0; k < 8; ++k) s += v[k];
        }
    add[y][x] = s;
    __syncthreads();
    if (y == 0 && col < a.width) {
        s = 0.0f;
#pragma unroll
        for (int r = 0; r < 32; ++r) s += add[r][x];
        out[col] = s;
    }
}

// Backward: threads of a row, and rows that a workgroup has at a time, by their width.  One workgroup a CU: its registers hold no second one of 512 threads, and fewer
// workgroups leave fewer parts to add (4096 x 4096, bf16, 201 MB: 39 us, 5.1 TB/s, and 5 to add the parts; in a form that took 48 + 5, twice as many workgroups took 53 + 7
// and two a CU at 128 registers, with spills, 91).  Beyond 4096 columns two units a thread: 4096 x 8192, fp16
// 83 us (403 MB, 4.9 TB/s), with biases 98; fp32 165 and, with some spills, 286.  (One unit in 1024 threads has half the registers a thread: 252 in fp16 without biases.)
static int row_threads(int width) { return width <= 512 ? 64 : width <= 1024 ? 128 : width <= 2048 ? 256 : 512; }
static int row_groups(int width) { return width <= 512 ? 8 : width <= 1024 ? 4 : width <= 2048 ? 2 : 1; }
static int64_t workgroups_of(int64_t rows, int32_t width) {
    const int64_t all = (rows + row_groups(width) - 1) / row_groups(width);
    return all < 256 ? all : 256;
}
// Whether a workgroup adds its groups' sums before it leaves them: where it has rows enough to pay for the barriers
static bool many_rows(int64_t rows, int32_t width) { return rows > 4 * workgroups_of(rows, width) * row_groups(width); }
static int64_t parts_of(int64_t rows, int32_t width) { return workgroups_of(rows, width) * (many_rows(rows, width) ? 1 : row_groups(width)); }
size_t residual_norm_partial_bytes(int64_t rows, int32_t width) {
    return align_up((size_t)parts_of(rows, width) * kGrads * (size_t)width * sizeof(float), 256);
}

// Whether a row's last thread may read eight columns whole: no output lies on what it reads, where a neighbour may have stored already.  Forward: f (and the weights), and x;
// backward: x, f, dh (and the weights), and dy.
template <int N> static bool may_read_whole(const ResidualNormArgs& a, const void* const (&read)[N], const void* out, const void* out_too) {
    bool apart = a.width >= 8;
    for (const void* p : read) apart = apart && p != out && p != out_too;
    return apart;
}

template <typename D, int TPR, int NV, int GROUPS> static hipError_t run_forward(ResidualNormArgs a, hipStream_t st) {
    a.whole = may_read_whole(a, {a.f}, a.y, a.h);
    a.whole_too = may_read_whole(a, {a.x}, a.y, a.h);
    const dim3 grid((unsigned)((a.rows + GROUPS - 1) / GROUPS)), block(TPR * GROUPS);
    if (a.drop.limit) hipLaunchKernelGGL((k_residual_norm<D, TPR, NV, GROUPS, true>), grid, block, 0, st, a);
    else hipLaunchKernelGGL((k_residual_norm<D, TPR, NV, GROUPS, false>), grid, block, 0, st, a);
    return hipGetLastError();
}
template <typename D, int TPR, int NV, int GROUPS> static hipError_t run_backward(ResidualNormArgs a, hipStream_t st) {
    const int64_t workgroups = workgroups_of(a.rows, a.width);
    a.many = many_rows(a.rows, a.width);
    a.whole = may_read_whole(a, {a.x, a.f, a.dh}, a.dx, a.df);
    a.whole_too = may_read_whole(a, {a.dy}, a.dx, a.df);
    const bool bias = (a.post != LSP_NORM_NONE && a.post_b) || a.grads[1] || a.grads[4];
    const dim3 grid((unsigned)workgroups), block(TPR * GROUPS);
    if (a.drop.limit && bias) hipLaunchKernelGGL((k_residual_norm_back<D, TPR, NV, GROUPS, true, true>), grid, block, 0, st, a);
    else if (a.drop.limit) hipLaunchKernelGGL((k_residual_norm_back<D, TPR, NV, GROUPS, true, false>), grid, block, 0, st, a);
    else if (bias) hipLaunchKernelGGL((k_residual_norm_back<D, TPR, NV, GROUPS, false, true>), grid, block, 0, st, a);
    else hipLaunchKernelGGL((k_residual_norm_back<D, TPR, NV, GROUPS, false, false>), grid, block, 0, st, a);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    int sums = 0;
    for (float* g : a.grads) sums += g != nullptr;
    if (!sums) return hipSuccess;
    hipLaunchKernelGGL(k_residual_norm_sums, dim3((unsigned)((a.width + 31) / 32), (unsigned)sums), dim3(1024), 0, st, a, (int)parts_of(a.rows, a.width));
    return hipGetLastError();
}

// Forward: a row has as few idle threads as the variants allow (3001 rows of 2999, fp16, dropout, 72 MB: 20.6 us, 3.5 TB/s; when this took 21.3, 256 threads of 16 columns in place of
// 128 of 24 took 22.8); beyond 4096 columns two units a thread in 512 threads (16384 rows of 8192, bf16, 1074 MB: 184 us, 5.8 TB/s; when this took 188, one unit in 1024 threads took
// 307, four in 256 threads 189).  Beside memory the vector units count: 45 instructions an element were all of their time, some 30 are left.
template <typename D> static hipError_t forward_of(const ResidualNormArgs& a, hipStream_t st) {
    if (a.width <= 64 * 8) return run_forward<D, 64, 1, 4>(a, st);
    if (a.width <= 64 * 16) return run_forward<D, 64, 2, 4>(a, st);
    if (a.width <= 64 * 24) return run_forward<D, 64, 3, 4>(a, st);
    if (a.width <= 256 * 8) return run_forward<D, 256, 1, 2>(a, st);
    if (a.width <= 128 * 24) return run_forward<D, 128, 3, 2>(a, st);
    if (a.width <= 256 * 16) return run_forward<D, 256, 2, 2>(a, st);
    return run_forward<D, 512, 2, 1>(a, st);
}
template <typename D> static hipError_t backward_of(const ResidualNormArgs& a, hipStream_t st) {
    switch (row_threads(a.width)) {
        case 64:  return run_backward<D, 64, 1, 8>(a, st);
        case 128: return run_backward<D, 128, 1, 4>(a, st);
        case 256: return run_backward<D, 256, 1, 2>(a, st);
        default:  return a.width <= 4096 ? run_backward<D, 512, 1, 1>(a, st) : run_backward<D, 512, 2, 1>(a, st);
    }
}

hipError_t launch_residual_norm_forward(const ResidualNormArgs& a, lsp_dtype dtype, hipStream_t st) {
    return dtype == LSP_F32 ? forward_of<F32>(a, st) : dtype == LSP_F16 ? forward_of<F16>(a, st) : forward_of<BF16>(a, st);
}
hipError_t launch_residual_norm_backward(const ResidualNormArgs& a, lsp_dtype dtype, hipStream_t st) {
    return dtype == LSP_F32 ? backward_of<F32>(a, st) : dtype == LSP_F16 ? backward_of<F16>(a, st) : backward_of<BF16>(a, st);
}

}  // namespace lsp

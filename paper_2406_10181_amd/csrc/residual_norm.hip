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
// Both are bound by memory: forward reads x and f and writes y and h, backward reads x, f, dy, dh and writes dx, df, each once.
#include "residual_norm.h"
#include "rows.h"

namespace lsp {

constexpr int kGrads = 5;

// Sums of N values over the TPR threads of a row, in all of them.  `scratch`: this row group's, two sets that take turns.
template <int TPR, int N> struct RowSum {
    float* scratch;                                       // LDS: [2][TPR / 64][N]
    int turn = 0;
    __device__ __forceinline__ void operator()(float (&v)[N]) {
#pragma unroll
        for (int s = 1; s < 64; s <<= 1)
#pragma unroll
            for (int k = 0; k < N; ++k) v[k] += __shfl_xor(v[k], s);
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

// mean and 1 / deviation of a row, by kind; v becomes (v - mean) / deviation
template <int TPR, int NV> __device__ __forceinline__ void normalise(Eight (&v)[NV], int kind, int width, float eps, int lane_col, RowSum<TPR, 1>& sum, float& mean, float& rstd) {
    mean = 0.0f; rstd = 1.0f;
    if (kind == LSP_NORM_NONE) return;
    const float per = 1.0f / (float)width;
    if (kind == LSP_NORM_LAYER) {
        float s[1] = {0.0f};
#pragma unroll
        for (int n = 0; n < NV; ++n)
#pragma unroll
            for (int e = 0; e < 8; ++e) s[0] += v[n].x[e];                                // (columns from width on are zeros)
        sum(s);
        mean = s[0] * per;
    }
    float s[1] = {0.0f};
#pragma unroll
    for (int n = 0; n < NV; ++n) {
        const int col = lane_col + n * TPR * 8;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float t = col + e < width ? v[n].x[e] - mean : 0.0f;
            s[0] = fmaf(t, t, s[0]);
            v[n].x[e] = t;
        }
    }
    sum(s);
    rstd = 1.0f / sqrtf(s[0] * per + eps);
#pragma unroll
    for (int n = 0; n < NV; ++n)
#pragma unroll
        for (int e = 0; e < 8; ++e) v[n].x[e] *= rstd;
}

template <typename D> __device__ __forceinline__ Eight vector_eight(const void* p, int col, int width, float otherwise) {
    if (!p) {
        Eight r;
#pragma unroll
        for (int e = 0; e < 8; ++e) r.x[e] = otherwise;
        return r;
    }
    return load_eight<D>(static_cast<const typename D::elem*>(p) + col, width - col);
}

template <typename D> __device__ __forceinline__ void drop_eight(Eight& v, int64_t row, int col, int width, const Dropout& drop) {
    const uint64_t n = (uint64_t)row * (uint64_t)((width + 7) >> 3) + (uint64_t)(col >> 3);
    const u32x4 w = philox((uint32_t)n, (uint32_t)(n >> 32), 0, drop.offset, drop.key0, drop.key1);
#pragma unroll
    for (int e = 0; e < 8; ++e) v.x[e] = philox_word(w, e) < drop.limit ? 0.0f : v.x[e] * drop.scale;
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
    Eight xv[NV], fv[NV];
#pragma unroll
    for (int n = 0; n < NV; ++n) {
        const int col = (t + n * TPR) * 8;
        xv[n] = load_eight<D>(x + col, width - col);
        fv[n] = load_eight<D>(f + col, width - col);
    }
    float mean_f, rstd_f, mean_y, rstd_y;
    normalise<TPR, NV>(fv, a.post, width, a.eps, t * 8, sum, mean_f, rstd_f);
#pragma unroll
    for (int n = 0; n < NV; ++n) {
        const int col = (t + n * TPR) * 8;
        if (a.post != LSP_NORM_NONE) {
            const Eight w = vector_eight<D>(a.post_w, col, width, 1.0f), b = vector_eight<D>(a.post_b, col, width, 0.0f);
#pragma unroll
            for (int e = 0; e < 8; ++e) fv[n].x[e] = fmaf(fv[n].x[e], w.x[e], b.x[e]);
        }
        if constexpr (DROP) drop_eight<D>(fv[n], row, col, width, a.drop);
        const Eight g = vector_eight<D>(a.gate, col, width, 1.0f);
#pragma unroll
        for (int e = 0; e < 8; ++e) xv[n].x[e] = col + e < width ? fmaf(a.branch_scale * g.x[e], fv[n].x[e], a.residual_scale * xv[n].x[e]) : 0.0f;
        if (mine) store_eight<D>(static_cast<elem*>(a.y) + row * a.y_stride + col, xv[n], width - col);
    }
    normalise<TPR, NV>(xv, a.pre, width, a.eps, t * 8, sum, mean_y, rstd_y);
    if (mine && a.h) {
#pragma unroll
        for (int n = 0; n < NV; ++n) {
            const int col = (t + n * TPR) * 8;
            if (a.pre != LSP_NORM_NONE) {
                const Eight w = vector_eight<D>(a.pre_w, col, width, 1.0f), b = vector_eight<D>(a.pre_b, col, width, 0.0f);
#pragma unroll
                for (int e = 0; e < 8; ++e) xv[n].x[e] = fmaf(xv[n].x[e], w.x[e], b.x[e]);
            }
            store_eight<D>(static_cast<elem*>(a.h) + row * a.h_stride + col, xv[n], width - col);
        }
    }
    if (mine && t == 0) {
        a.stats[row] = mean_f; a.stats[a.rows + row] = rstd_f;
        a.stats[2 * a.rows + row] = mean_y; a.stats[3 * a.rows + row] = rstd_y;
    }
}

template <typename D, int TPR, int NV, int GROUPS, bool DROP>
__global__ __launch_bounds__(TPR * GROUPS) void k_residual_norm_back(const ResidualNormArgs a) {
    using elem = typename D::elem;
    __shared__ float scratch[GROUPS][2 * 2 * (TPR / 64)];
    const int group = threadIdx.x / TPR, t = threadIdx.x % TPR;
    const int width = a.width;
    const float per = 1.0f / (float)width;
    RowSum<TPR, 2> sum{scratch[group]};
    float acc[kGrads][NV][8];
#pragma unroll
    for (int k = 0; k < kGrads; ++k)
#pragma unroll
        for (int n = 0; n < NV; ++n)
#pragma unroll
            for (int e = 0; e < 8; ++e) acc[k][n][e] = 0.0f;
    const int64_t step = (int64_t)gridDim.x * GROUPS;
    for (int64_t base = (int64_t)blockIdx.x * GROUPS; base < a.rows; base += step) {
        const bool mine = base + group < a.rows;
        const int64_t row = mine ? base + group : a.rows - 1;
        const elem* x = static_cast<const elem*>(a.x) + row * a.x_stride;
        const elem* f = static_cast<const elem*>(a.f) + row * a.f_stride;
        const elem* dy = static_cast<const elem*>(a.dy) + row * a.dy_stride;
        const elem* dh = a.dh ? static_cast<const elem*>(a.dh) + row * a.dh_stride : nullptr;
        Eight xv[NV], fv[NV], dyv[NV], dhv[NV];
#pragma unroll
        for (int n = 0; n < NV; ++n) {
            const int col = (t + n * TPR) * 8;
            xv[n] = load_eight<D>(x + col, width - col);
            fv[n] = load_eight<D>(f + col, width - col);
            dyv[n] = load_eight<D>(dy + col, width - col);
            if (dh) dhv[n] = load_eight<D>(dh + col, width - col);
            else
#pragma unroll
                for (int e = 0; e < 8; ++e) dhv[n].x[e] = 0.0f;
        }
        const float mean_f = a.stats[row], rstd_f = a.stats[a.rows + row], mean_y = a.stats[2 * a.rows + row], rstd_y = a.stats[3 * a.rows + row];
        float s[2] = {0.0f, 0.0f};
        // xv: y^, dhv: the gradient of y^;  fv: f^
        uint32_t kept[NV];
#pragma unroll
        for (int n = 0; n < NV; ++n) {
            const int col = (t + n * TPR) * 8;
            Eight u;
#pragma unroll
            for (int e = 0; e < 8; ++e) { fv[n].x[e] = col + e < width ? (fv[n].x[e] - mean_f) * rstd_f : 0.0f; u.x[e] = fv[n].x[e]; }
            if (a.post != LSP_NORM_NONE) {
                const Eight w = vector_eight<D>(a.post_w, col, width, 1.0f), b = vector_eight<D>(a.post_b, col, width, 0.0f);
#pragma unroll
                for (int e = 0; e < 8; ++e) u.x[e] = fmaf(u.x[e], w.x[e], b.x[e]);
            }
            kept[n] = 0xFFu;
            if constexpr (DROP) {
                const uint64_t at = (uint64_t)row * (uint64_t)((width + 7) >> 3) + (uint64_t)(col >> 3);
                const u32x4 w = philox((uint32_t)at, (uint32_t)(at >> 32), 0, a.drop.offset, a.drop.key0, a.drop.key1);
                kept[n] = 0;
#pragma unroll
                for (int e = 0; e < 8; ++e) kept[n] |= (philox_word(w, e) < a.drop.limit ? 0u : 1u) << e;
            }
            const Eight g = vector_eight<D>(a.gate, col, width, 1.0f), wp = vector_eight<D>(a.pre != LSP_NORM_NONE ? a.pre_w : nullptr, col, width, 1.0f);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float keep = !DROP ? 1.0f : (kept[n] >> e) & 1u ? a.drop.scale : 0.0f;
                const float kept_u = keep == 0.0f ? 0.0f : keep * u.x[e];                 // (what is dropped may be infinite)
                const float y = fmaf(a.branch_scale * g.x[e], kept_u, a.residual_scale * xv[n].x[e]);
                const float hat = col + e < width ? (y - mean_y) * rstd_y : 0.0f;
                const float d = dhv[n].x[e];
                if (mine) { acc[0][n][e] = fmaf(d, hat, acc[0][n][e]); acc[1][n][e] += d; }
                const float de = d * wp.x[e];
                xv[n].x[e] = hat;
                dhv[n].x[e] = de;
                s[0] = fmaf(de, hat, s[0]);
                s[1] += de;
            }
        }
        if (a.pre != LSP_NORM_NONE) sum(s);
        float s1 = s[0] * per, s0 = a.pre == LSP_NORM_LAYER ? s[1] * per : 0.0f;
        s[0] = s[1] = 0.0f;
#pragma unroll
        for (int n = 0; n < NV; ++n) {
            const int col = (t + n * TPR) * 8;
            Eight out;
            const Eight g = vector_eight<D>(a.gate, col, width, 1.0f);
            const Eight w = vector_eight<D>(a.post != LSP_NORM_NONE ? a.post_w : nullptr, col, width, 1.0f), b = vector_eight<D>(a.post != LSP_NORM_NONE ? a.post_b : nullptr, col, width, 0.0f);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float total = dyv[n].x[e] + (a.pre == LSP_NORM_NONE ? dhv[n].x[e] : rstd_y * (dhv[n].x[e] - s0 - xv[n].x[e] * s1));
                out.x[e] = a.residual_scale * total;
                const float keep = !DROP ? 1.0f : (kept[n] >> e) & 1u ? a.drop.scale : 0.0f;
                const float branch = a.branch_scale * total * keep, u = keep == 0.0f ? 0.0f : fmaf(fv[n].x[e], w.x[e], b.x[e]);
                const float du = branch * g.x[e];
                if (mine) {
                    acc[2][n][e] = fmaf(branch, u, acc[2][n][e]);
                    acc[3][n][e] = fmaf(du, fv[n].x[e], acc[3][n][e]);
                    acc[4][n][e] += du;
                }
                const float de = col + e < width ? du * w.x[e] : 0.0f;
                dyv[n].x[e] = de;
                s[0] = fmaf(de, fv[n].x[e], s[0]);
                s[1] += de;
            }
            if (mine) store_eight<D>(static_cast<elem*>(a.dx) + row * a.dx_stride + col, out, width - col);
        }
        if (a.post != LSP_NORM_NONE) sum(s);
        s1 = s[0] * per; s0 = a.post == LSP_NORM_LAYER ? s[1] * per : 0.0f;
#pragma unroll
        for (int n = 0; n < NV; ++n) {
            const int col = (t + n * TPR) * 8;
            Eight out;
#pragma unroll
            for (int e = 0; e < 8; ++e) out.x[e] = a.post == LSP_NORM_NONE ? dyv[n].x[e] : rstd_f * (dyv[n].x[e] - s0 - fv[n].x[e] * s1);
            if (mine) store_eight<D>(static_cast<elem*>(a.df) + row * a.df_stride + col, out, width - col);
        }
    }
    // this row group's part of the sums over rows
    const int64_t part = (int64_t)blockIdx.x * GROUPS + group, parts = (int64_t)gridDim.x * GROUPS;
    int slot = 0;
#pragma unroll
    for (int k = 0; k < kGrads; ++k) {
        if (!a.grads[k]) continue;
        float* out = a.partial + ((int64_t)slot * parts + part) * width;
        ++slot;
#pragma unroll
        for (int n = 0; n < NV; ++n) {
            const int col = (t + n * TPR) * 8;
            Eight v;
#pragma unroll
            for (int e = 0; e < 8; ++e) v.x[e] = acc[k][n][e];
            store_eight<F32>(out + col, v, width - col);
        }
    }
}

// Adds the parts: a workgroup has 64 columns of one sum, its four waves take turns at the parts.
__global__ __launch_bounds__(256) void k_residual_norm_sums(const ResidualNormArgs a, int64_t parts) {
    __shared__ float add[4][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int col = blockIdx.x * 64 + lane;
    float* out = nullptr;
    int slot = 0;
#pragma unroll
    for (int k = 0; k < kGrads; ++k)
        if (a.grads[k]) { if (slot == (int)blockIdx.y) out = a.grads[k]; ++slot; }
    const float* p = a.partial + (int64_t)blockIdx.y * parts * a.width;
    float s = 0.0f;
    if (col < a.width)
        for (int64_t r = wave; r < parts; r += 4) s += p[r * a.width + col];
    add[wave][lane] = s;
    __syncthreads();
    if (wave == 0 && col < a.width) out[col] = (add[0][lane] + add[1][lane]) + (add[2][lane] + add[3][lane]);
}

// Rows that a workgroup has at a time, by their width
static int groups_of(int width) { return width <= 1024 ? 4 : width <= 4096 ? 2 : 1; }

static int64_t workgroups_of(int64_t rows, int32_t width) {
    const int64_t all = (rows + groups_of(width) - 1) / groups_of(width);
    return all < 256 ? all : 256;
}
size_t residual_norm_partial_bytes(int64_t rows, int32_t width) {
    return align_up((size_t)workgroups_of(rows, width) * groups_of(width) * kGrads * (size_t)width * sizeof(float), 256);
}

template <typename D, int TPR, int NV, int GROUPS> static hipError_t run_forward(const ResidualNormArgs& a, hipStream_t st) {
    const dim3 grid((unsigned)((a.rows + GROUPS - 1) / GROUPS)), block(TPR * GROUPS);
    if (a.drop.limit) hipLaunchKernelGGL((k_residual_norm<D, TPR, NV, GROUPS, true>), grid, block, 0, st, a);
    else hipLaunchKernelGGL((k_residual_norm<D, TPR, NV, GROUPS, false>), grid, block, 0, st, a);
    return hipGetLastError();
}
template <typename D, int TPR, int NV, int GROUPS> static hipError_t run_backward(const ResidualNormArgs& a, hipStream_t st) {
    const int64_t workgroups = workgroups_of(a.rows, a.width);
    if (a.drop.limit) hipLaunchKernelGGL((k_residual_norm_back<D, TPR, NV, GROUPS, true>), dim3((unsigned)workgroups), dim3(TPR * GROUPS), 0, st, a);
    else hipLaunchKernelGGL((k_residual_norm_back<D, TPR, NV, GROUPS, false>), dim3((unsigned)workgroups), dim3(TPR * GROUPS), 0, st, a);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    int sums = 0;
    for (float* g : a.grads) sums += g != nullptr;
    if (!sums) return hipSuccess;
    hipLaunchKernelGGL(k_residual_norm_sums, dim3((unsigned)((a.width + 63) / 64), (unsigned)sums), dim3(256), 0, st, a, workgroups * GROUPS);
    return hipGetLastError();
}

template <typename D> static hipError_t forward_of(const ResidualNormArgs& a, hipStream_t st) {
    if (a.width <= 512) return run_forward<D, 64, 1, 4>(a, st);
    if (a.width <= 1024) return run_forward<D, 64, 2, 4>(a, st);
    if (a.width <= 2048) return run_forward<D, 256, 1, 2>(a, st);
    if (a.width <= 4096) return run_forward<D, 256, 2, 2>(a, st);
    return run_forward<D, 512, 2, 1>(a, st);
}
template <typename D> static hipError_t backward_of(const ResidualNormArgs& a, hipStream_t st) {
    if (a.width <= 512) return run_backward<D, 64, 1, 4>(a, st);
    if (a.width <= 1024) return run_backward<D, 64, 2, 4>(a, st);
    if (a.width <= 2048) return run_backward<D, 256, 1, 2>(a, st);
    if (a.width <= 4096) return run_backward<D, 256, 2, 2>(a, st);
    return run_backward<D, 512, 2, 1>(a, st);
}

hipError_t launch_residual_norm_forward(const ResidualNormArgs& a, lsp_dtype dtype, hipStream_t st) {
    return dtype == LSP_F32 ? forward_of<F32>(a, st) : dtype == LSP_F16 ? forward_of<F16>(a, st) : forward_of<BF16>(a, st);
}
hipError_t launch_residual_norm_backward(const ResidualNormArgs& a, lsp_dtype dtype, hipStream_t st) {
    return dtype == LSP_F32 ? backward_of<F32>(a, st) : dtype == LSP_F16 ? backward_of<F16>(a, st) : backward_of<BF16>(a, st);
}

}  // namespace lsp

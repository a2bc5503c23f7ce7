// Norms of query and key heads with the rotation by position, and back; keys and values may go straight to their places in a cache.
//
// Bound by memory: a head is read and written once (backward: its gradient read, what was normed read again, a gradient written).  A group of 4, 8 or 16 lanes has a
// head, eight elements a lane, so that the sums of a norm go through the lanes of a group by moves that need no LDS.  A lane's eight elements are four
// whole pairs: four elements from each half of what turns, or eight neighbours; so turning needs no other lane, and the lane's four angles are the same
// for every head of a token.  They cost an fp64 product and a sine and cosine each, some 200 instructions; a group keeps them for all rows of the token that it does.
// Where there are few tokens their rows are dealt to many groups (`parts`), since then the angles are not what takes the time.
#include <algorithm>

#include "rotary.h"
#include "rows.h"

namespace lsp {

constexpr int kRotaryThreads = 256;

// Sum over GROUP lanes, in all of them: within four and eight and sixteen by permutations of the lanes of a row
template <int CTRL> __device__ __forceinline__ float with_lane(float x) {
    return x + __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), CTRL, 0xF, 0xF, false));
}
template <int GROUP> __device__ __forceinline__ float group_sum(float x) {
    x = with_lane<0xB1>(x); x = with_lane<0x4E>(x);                      // lane ^ 1, lane ^ 2
    if constexpr (GROUP >= 8) x = with_lane<0x141>(x);                   // the other four of eight (mirrored)
    if constexpr (GROUP >= 16) x = with_lane<0x140>(x);                  // the other eight of sixteen
    return x;
}

// Where a lane's two fours of a head lie, and which angles are its own
struct Place {
    int first, second, pair;                      // elements; first pair, or -1: what stays
    bool there;
    __device__ __forceinline__ Place(const RotaryArgs& a, int lane) {
        const int half = a.rotated / 2;
        there = lane * 8 < a.head_dim;
        pair = lane * 4 < half ? lane * 4 : -1;
        first = pair >= 0 && !a.neighbours ? pair : lane * 8;
        second = pair >= 0 && !a.neighbours ? half + pair : lane * 8 + 4;
    }
};

template <typename D> struct Raw { u32x4 a, b; };                        // 16 bits: the first two words of each
template <typename D> __device__ __forceinline__ Raw<D> load_raw(const uint8_t* row, const Place& at) {
    Raw<D> r;
    if constexpr (D::size == 4) {
        r.a = *reinterpret_cast<const u32x4*>(row + at.first * 4);
        r.b = *reinterpret_cast<const u32x4*>(row + at.second * 4);
    } else {
        const u32x2 x = *reinterpret_cast<const u32x2*>(row + at.first * 2), y = *reinterpret_cast<const u32x2*>(row + at.second * 2);
        r.a[0] = x[0]; r.a[1] = x[1]; r.b[0] = y[0]; r.b[1] = y[1];
    }
    return r;
}
template <typename D> __device__ __forceinline__ Eight widen_raw(const Raw<D>& r) {
    Packed<D> p;
#pragma unroll
    for (int k = 0; k < D::size; ++k) { p.w[k] = r.a[k]; p.w[D::size + k] = r.b[k]; }
    return widen_eight<D>(p);
}
template <typename D> __device__ __forceinline__ void store_raw(uint8_t* row, const Place& at, const Eight& x) {
    const Packed<D> o = narrow_eight<D>(x);
    if constexpr (D::size == 4) {
        *reinterpret_cast<u32x4*>(row + at.first * 4) = u32x4{o.w[0], o.w[1], o.w[2], o.w[3]};
        *reinterpret_cast<u32x4*>(row + at.second * 4) = u32x4{o.w[4], o.w[5], o.w[6], o.w[7]};
    } else {
        *reinterpret_cast<u32x2*>(row + at.first * 2) = u32x2{o.w[0], o.w[1]};
        *reinterpret_cast<u32x2*>(row + at.second * 2) = u32x2{o.w[2], o.w[3]};
    }
}
template <typename D> __device__ __forceinline__ Eight load_vector(const void* v, const Place& at, float otherwise) {
    Eight r;
#pragma unroll
    for (int e = 0; e < 8; ++e) r.x[e] = otherwise;
    if (v && at.there) r = widen_raw<D>(load_raw<D>(static_cast<const uint8_t*>(v), at));
    return r;
}

struct Angles { float cos[4], sin[4]; };
// Whole turns are taken off in fp64: position and frequency have 55 bits together at most, and what is left of a turn keeps at least 30 behind the point
__device__ __forceinline__ Angles angles_of(const float (&frequency)[4], int64_t position, bool turns) {
    Angles r;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        r.cos[j] = 1.0f; r.sin[j] = 0.0f;
        if (!turns) continue;
        const double whole = (double)position * ((double)frequency[j] * 0.15915494309189533577);
        sincospif(2.0f * (float)(whole - rint(whole)), &r.sin[j], &r.cos[j]);
    }
    return r;
}
// BACK: by minus the angle
template <bool NEIGHBOURS, bool BACK> __device__ __forceinline__ void turn(Eight& x, const Angles& t) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        float& a = x.x[NEIGHBOURS ? 2 * j : j];
        float& b = x.x[NEIGHBOURS ? 2 * j + 1 : 4 + j];
        const float s = BACK ? -t.sin[j] : t.sin[j], u = a, v = b;
        a = u * t.cos[j] - v * s;
        b = u * s + v * t.cos[j];
    }
}

// Whether the token counts, its position and the place of its key
struct Token { int text, i; int64_t position, place; bool counts; };
__device__ __forceinline__ Token token_of(const RotaryArgs& a, int token) {
    Token t;
    t.text = token / a.length;
    t.i = token - t.text * a.length;
    t.counts = t.i < valid_length(a.lens, t.text, a.length);
    t.place = t.position = (int64_t)t.i + (a.starts ? a.starts[t.text] : 0);
    if (a.positions && t.counts) t.position = a.positions[(int64_t)t.text * a.length + t.i];
    return t;
}

template <int NORM, int GROUP> __device__ __forceinline__ void norm_head(Eight& x, float& factor, const Place& at, int head_dim, float eps) {
    factor = 1.0f;
    if constexpr (NORM != LSP_NORM_NONE) {
        const float share = 1.0f / (float)head_dim;
        if constexpr (NORM == LSP_NORM_LAYER) {
            float sum = 0.0f;
#pragma unroll
            for (int e = 0; e < 8; ++e) sum += x.x[e];
            const float mean = group_sum<GROUP>(sum) * share;
#pragma unroll
            for (int e = 0; e < 8; ++e) x.x[e] = at.there ? x.x[e] - mean : 0.0f;
        }
        float squares = 0.0f;
#pragma unroll
        for (int e = 0; e < 8; ++e) squares = fmaf(x.x[e], x.x[e], squares);
        factor = 1.0f / sqrtf(fmaf(group_sum<GROUP>(squares), share, eps));
#pragma unroll
        for (int e = 0; e < 8; ++e) x.x[e] *= factor;
    }
}

constexpr int kAtOnce = 4;                          // rows whose loads are on their way together

template <typename D, int NORM, int GROUP, bool NEIGHBOURS>
__global__ __launch_bounds__(kRotaryThreads) void k_rotary(RotaryArgs a) {
    const int lane = threadIdx.x % GROUP;
    const int64_t group = (int64_t)blockIdx.x * (kRotaryThreads / GROUP) + threadIdx.x / GROUP;
    if (group >= (int64_t)a.batch * a.length * a.parts) return;
    const int token = (int)(group / a.parts), part = (int)(group - (int64_t)token * a.parts);
    const Token t = token_of(a, token);
    if (!t.counts) return;
    const Place at(a, lane);
    const bool inside = t.place >= 0 && t.place < a.cache;
    // the row and its destination; NULL: nowhere
    const auto from = [&](int row) -> const uint8_t* {
        if (!at.there) return nullptr;
        if (row < a.heads) return lsp::at<D>(a.q, t.text, t.i, row);
        if (!inside) return nullptr;
        return row < a.heads + a.kv_heads ? lsp::at<D>(a.k, t.text, t.i, row - a.heads) : lsp::at<D>(a.v, t.text, t.i, row - a.heads - a.kv_heads);
    };
    const auto to = [&](int row) -> uint8_t* {
        const uint8_t* p = row < a.heads ? lsp::at<D>(a.qr, t.text, t.i, row)
                         : row < a.heads + a.kv_heads ? lsp::at<D>(a.kr, t.text, t.place, row - a.heads) : lsp::at<D>(a.vr, t.text, t.place, row - a.heads - a.kv_heads);
        return const_cast<uint8_t*>(p);
    };
    const auto fetch = [&](int row) {
        Raw<D> r;
        r.a = r.b = u32x4{0, 0, 0, 0};
        const uint8_t* p = row < a.rows ? from(row) : nullptr;
        if (p) r = load_raw<D>(p, at);
        return r;
    };
    Raw<D> raw[kAtOnce];
#pragma unroll
    for (int k = 0; k < kAtOnce; ++k) raw[k] = fetch(part + k * a.parts);
    float frequency[4] = {0.0f, 0.0f, 0.0f, 0.0f};
    if (at.pair >= 0) {
#pragma unroll
        for (int j = 0; j < 4; ++j) frequency[j] = a.frequencies[at.pair + j];
    }
    const Eight qw = load_vector<D>(a.q_w, at, 1.0f), kw = load_vector<D>(a.k_w, at, 1.0f), qb = load_vector<D>(a.q_b, at, 0.0f), kb = load_vector<D>(a.k_b, at, 0.0f);
    const Angles angles = angles_of(frequency, t.position, at.pair >= 0);
    for (int row0 = part; row0 < a.rows; row0 += kAtOnce * a.parts) {
        Raw<D> next[kAtOnce];
#pragma unroll
        for (int k = 0; k < kAtOnce; ++k) next[k] = fetch(row0 + (kAtOnce + k) * a.parts);
#pragma unroll
        for (int k = 0; k < kAtOnce; ++k) {
            const int row = row0 + k * a.parts;
            if (row >= a.rows) break;                                    // (the same for a group's lanes)
            Eight x = widen_raw<D>(raw[k]);
            if (row < a.heads + a.kv_heads) {
                const bool query = row < a.heads;
                float factor;
                norm_head<NORM, GROUP>(x, factor, at, a.head_dim, a.eps);
                if constexpr (NORM != LSP_NORM_NONE) {
#pragma unroll
                    for (int e = 0; e < 8; ++e) x.x[e] = fmaf(x.x[e], query ? qw.x[e] : kw.x[e], query ? qb.x[e] : kb.x[e]);
                }
                turn<NEIGHBOURS, false>(x, angles);
            }
            if (at.there && (row < a.heads || inside)) store_raw<D>(to(row), at, x);
        }
#pragma unroll
        for (int k = 0; k < kAtOnce; ++k) raw[k] = next[k];
    }
}

// With y = xhat w + b turned by the angle, and d the gradient of the result turned back:  dw += d xhat, db += d, and with e = d w
//   dx = factor (e - xhat mean(e xhat) [- mean(e), for a norm with means]).
template <typename D, int NORM, int GROUP, bool NEIGHBOURS>
__global__ __launch_bounds__(kRotaryThreads) void k_rotary_back(RotaryArgs a) {
    constexpr int kGroups = kRotaryThreads / GROUP;
    const int lane = threadIdx.x % GROUP, own = threadIdx.x / GROUP;
    const Place at(a, lane);
    float frequency[4] = {0.0f, 0.0f, 0.0f, 0.0f};
    if (at.pair >= 0) {
#pragma unroll
        for (int j = 0; j < 4; ++j) frequency[j] = a.frequencies[at.pair + j];
    }
    const Eight qw = load_vector<D>(a.q_w, at, 1.0f), kw = load_vector<D>(a.k_w, at, 1.0f);
    float sums[4][8];                                                    // of q_weight, k_weight, q_bias, k_bias
#pragma unroll
    for (int s = 0; s < 4; ++s)
#pragma unroll
        for (int e = 0; e < 8; ++e) sums[s][e] = 0.0f;
    const int64_t items = (int64_t)a.batch * a.length * a.parts;
    for (int64_t item = (int64_t)blockIdx.x * kGroups + own; item < items; item += (int64_t)a.blocks * kGroups) {
        const int token = (int)(item / a.parts), part = (int)(item - (int64_t)token * a.parts);
        const Token t = token_of(a, token);
        const bool inside = t.place >= 0 && t.place < a.cache;
        const Angles angles = angles_of(frequency, t.position, at.pair >= 0);
        for (int row = part; row < a.rows; row += a.parts) {
            const bool query = row < a.heads;
            const int head = query ? row : row - a.heads;
            const bool seen = t.counts && (query || inside) && at.there;
            Eight d, x;
#pragma unroll
            for (int e = 0; e < 8; ++e) d.x[e] = x.x[e] = 0.0f;
            if (seen) {
                d = widen_raw<D>(load_raw<D>(query ? lsp::at<D>(a.qr, t.text, t.i, head) : lsp::at<D>(a.kr, t.text, t.place, head), at));
                if constexpr (NORM != LSP_NORM_NONE) x = widen_raw<D>(load_raw<D>(query ? lsp::at<D>(a.q, t.text, t.i, head) : lsp::at<D>(a.k, t.text, t.i, head), at));
            }
            turn<NEIGHBOURS, true>(d, angles);
            if constexpr (NORM != LSP_NORM_NONE) {
                float factor;
                norm_head<NORM, GROUP>(x, factor, at, a.head_dim, a.eps);
                float along = 0.0f, sum = 0.0f;
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const float dw = d.x[e] * x.x[e];
                    sums[0][e] += query ? dw : 0.0f; sums[1][e] += query ? 0.0f : dw;
                    sums[2][e] += query ? d.x[e] : 0.0f; sums[3][e] += query ? 0.0f : d.x[e];
                    d.x[e] *= query ? qw.x[e] : kw.x[e];
                    along = fmaf(d.x[e], x.x[e], along);
                    sum += d.x[e];
                }
                const float share = 1.0f / (float)a.head_dim;
                along = group_sum<GROUP>(along) * share;
                const float mean = NORM == LSP_NORM_LAYER ? group_sum<GROUP>(sum) * share : 0.0f;
#pragma unroll
                for (int e = 0; e < 8; ++e) d.x[e] = seen ? factor * (d.x[e] - fmaf(x.x[e], along, mean)) : 0.0f;
            }
            if (at.there) store_raw<D>(const_cast<uint8_t*>(query ? lsp::at<D>(a.v, t.text, t.i, head) : lsp::at<D>(a.vr, t.text, t.i, head)), at, d);
        }
    }
    if (NORM == LSP_NORM_NONE || !a.sums) return;
    __shared__ float all[kGroups][GROUP * 8 + 4];
#pragma unroll
    for (int s = 0; s < 4; ++s) {
        __syncthreads();
        if (at.there) {
#pragma unroll
            for (int e = 0; e < 8; ++e) all[own][e < 4 ? at.first + e : at.second + e - 4] = sums[s][e];
        }
        __syncthreads();
        if ((int)threadIdx.x < a.head_dim) {
            float x = 0.0f;
#pragma unroll
            for (int g = 0; g < kGroups; ++g) x += all[g][threadIdx.x];
            a.partial[((int64_t)blockIdx.x * 4 + s) * a.head_dim + threadIdx.x] = x;
        }
    }
}

// The workgroups' parts of a sum, added in their order: 16 columns of one sum a workgroup, 16 runs of parts side by side
__global__ __launch_bounds__(256) void k_rotary_sums(RotaryArgs a) {
    const int s = blockIdx.y, column = blockIdx.x * 16 + (threadIdx.x & 15), run = threadIdx.x >> 4;
    float* const to = a.grads[s];
    if (!to) return;
    float x = 0.0f;
    if (column < a.head_dim) {
#pragma unroll 4
        for (int p = run; p < a.blocks; p += 16) x += a.partial[((int64_t)p * 4 + s) * a.head_dim + column];
    }
    __shared__ float all[16][17];
    all[run][threadIdx.x & 15] = x;
    __syncthreads();
    if (run == 0 && column < a.head_dim) {
        float sum = 0.0f;
#pragma unroll
        for (int r = 0; r < 16; ++r) sum += all[r][threadIdx.x & 15];
        to[column] = sum;
    }
}

static int group_of(int head_dim) { return head_dim <= 32 ? 4 : head_dim <= 64 ? 8 : 16; }

void plan_rotary(RotaryArgs& a, bool backward) {
    const int64_t tokens = (int64_t)a.batch * a.length;
    const int per_block = kRotaryThreads / group_of(a.head_dim);
    // lane groups for 2048 workgroups, as far as there are rows
    a.parts = (int)std::min<int64_t>(a.rows, std::max<int64_t>(1, (2048 * per_block + tokens - 1) / tokens));
    const int64_t blocks = (tokens * a.parts + per_block - 1) / per_block;
    a.blocks = (int)(backward && a.sums ? std::min<int64_t>(blocks, 1024) : blocks);
}
size_t rotary_partial_bytes(const RotaryArgs& a) { return a.sums ? align_up((size_t)a.blocks * 4 * a.head_dim * sizeof(float), 256) : 0; }

template <typename D, int NORM, int GROUP> static void launch_one(const RotaryArgs& a, bool backward, hipStream_t st) {
    const dim3 grid((unsigned)a.blocks), block(kRotaryThreads);
    if (backward) {
        if (a.neighbours) hipLaunchKernelGGL((k_rotary_back<D, NORM, GROUP, true>), grid, block, 0, st, a);
        else hipLaunchKernelGGL((k_rotary_back<D, NORM, GROUP, false>), grid, block, 0, st, a);
    } else {
        if (a.neighbours) hipLaunchKernelGGL((k_rotary<D, NORM, GROUP, true>), grid, block, 0, st, a);
        else hipLaunchKernelGGL((k_rotary<D, NORM, GROUP, false>), grid, block, 0, st, a);
    }
}
template <typename D, int NORM> static void launch_group(const RotaryArgs& a, bool backward, hipStream_t st) {
    const int group = group_of(a.head_dim);
    if (group == 4) launch_one<D, NORM, 4>(a, backward, st);
    else if (group == 8) launch_one<D, NORM, 8>(a, backward, st);
    else launch_one<D, NORM, 16>(a, backward, st);
}
template <typename D> static void launch_norm(const RotaryArgs& a, bool backward, hipStream_t st) {
    if (a.norm == LSP_NORM_NONE) launch_group<D, LSP_NORM_NONE>(a, backward, st);
    else if (a.norm == LSP_NORM_RMS) launch_group<D, LSP_NORM_RMS>(a, backward, st);
    else launch_group<D, LSP_NORM_LAYER>(a, backward, st);
}

hipError_t launch_rotary(const RotaryArgs& a, bool backward, lsp_dtype dtype, hipStream_t st) {
    if (dtype == LSP_F32) launch_norm<F32>(a, backward, st);
    else if (dtype == LSP_F16) launch_norm<F16>(a, backward, st);
    else launch_norm<BF16>(a, backward, st);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || !backward || !a.sums) return e;
    hipLaunchKernelGGL(k_rotary_sums, dim3((unsigned)((a.head_dim + 15) / 16), 4), dim3(256), 0, st, a);
    return hipGetLastError();
}

}  // namespace lsp

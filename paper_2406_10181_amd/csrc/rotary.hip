// Norms of query and key heads with the rotation by position, and back; keys and values may go straight to their places in a cache.
//
// Bound by memory: a head is read and written once (backward: its gradient read, what was normed read again, a gradient written).  A group of 4, 8 or 16 lanes has a
// head, eight elements a lane, so that the sums of a norm go through the lanes of a group by moves that need no LDS.  A lane's eight elements are four
// whole pairs: four elements from each half of what turns, or eight neighbours; so turning needs no other lane.  A wave has 4, 8 or 16 heads of one token at a time, whose addresses are a scalar
// base and what the lane adds to it once (with addresses of its own for every head a lane spent 240 instructions on one in the backward pass).  A workgroup has the queries, the keys
// or the values of a few tokens that follow one another; its angles, some products in fp64, a sine and a cosine each, are made once for all their heads and lie in LDS.
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
// Bytes from a base to a lane's two fours
struct Reach { uint32_t first, second; };
template <typename D> __device__ __forceinline__ Raw<D> load_raw(const uint8_t* base, const Reach& at) {
    Raw<D> r;
    if constexpr (D::size == 4) {
        r.a = *reinterpret_cast<const u32x4*>(base + at.first);
        r.b = *reinterpret_cast<const u32x4*>(base + at.second);
    } else {
        const u32x2 x = *reinterpret_cast<const u32x2*>(base + at.first), y = *reinterpret_cast<const u32x2*>(base + at.second);
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
template <typename D> __device__ __forceinline__ void store_raw(uint8_t* base, const Reach& at, const Eight& x) {
    const Packed<D> o = narrow_eight<D>(x);
    if constexpr (D::size == 4) {
        *reinterpret_cast<u32x4*>(base + at.first) = u32x4{o.w[0], o.w[1], o.w[2], o.w[3]};
        *reinterpret_cast<u32x4*>(base + at.second) = u32x4{o.w[4], o.w[5], o.w[6], o.w[7]};
    } else {
        *reinterpret_cast<u32x2*>(base + at.first) = u32x2{o.w[0], o.w[1]};
        *reinterpret_cast<u32x2*>(base + at.second) = u32x2{o.w[2], o.w[3]};
    }
}
// `head`: the lane's, of those that its wave has at a time
template <typename D> __device__ __forceinline__ Reach reach_of(const Place& at, const Strided& s, int head) {
    const uint32_t begin = (uint32_t)(head * s.head) * D::size;
    return {begin + at.first * D::size, begin + at.second * D::size};
}
template <typename D> __device__ __forceinline__ Eight load_vector(const void* v, const Place& at, float otherwise) {
    Eight r;
#pragma unroll
    for (int e = 0; e < 8; ++e) r.x[e] = otherwise;
    if (v && at.there) r = widen_raw<D>(load_raw<D>(static_cast<const uint8_t*>(v), Reach{(uint32_t)at.first * D::size, (uint32_t)at.second * D::size}));
    return r;
}

// By the angle, or (BACK) by minus the angle
template <bool NEIGHBOURS, bool BACK> __device__ __forceinline__ void turn(Eight& x, const f32x4& cos, const f32x4& sin) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        float& a = x.x[NEIGHBOURS ? 2 * j : j];
        float& b = x.x[NEIGHBOURS ? 2 * j + 1 : 4 + j];
        const float s = BACK ? -sin[j] : sin[j], u = a, v = b;
        a = u * cos[j] - v * s;
        b = u * s + v * cos[j];
    }
}

// The tokens of a workgroup, in LDS
struct Tokens {
    float   cos[kRotaryTokens][LSP_MAX_HEAD_DIM / 2], sin[kRotaryTokens][LSP_MAX_HEAD_DIM / 2];
    int64_t x[kRotaryTokens], y[kRotaryTokens], out[kRotaryTokens];      // elements from the tensors' begins to the token's first head; -1: not there
    int64_t position[kRotaryTokens];
};
// Turns of an angle that is position * frequency.  One over 2 pi comes in two parts, and what each product's rounding takes off is added: a product of 2^31 alone would be off by 2^-23 of a turn, this is by
// 2^-53 up to 2^51 and by 2^-35 at 2^71 radians.  (Contracted, turns - rint(turns) would have the product without its rounding, and that would count twice.)  Whole turns and then quarters are taken off in
// fp64, so that fp32 has 1/8 of a turn at most, off by 2^-28: there Taylor's series of five and six terms leave 0.1 EPS, and sine and cosine are off by 2.8 and 1.8 EPS at most (EPS = 2^-24; the library's
// sincospif, with quarters of its own: 2 heads of 128 over 11720 tokens 4 % longer).
__device__ __forceinline__ void sine_and_cosine(int64_t position, float frequency, float& sin, float& cos) {
#pragma clang fp contract(off)
    constexpr double kPerRadian = 0.15915494309189535, kRest = -9.839338337591243e-18;
    const double f = (double)frequency, p = (double)position;
    const double each = f * kPerRadian, each_rest = fma(f, kPerRadian, -each) + f * kRest;
    const double turns = p * each, rest = fma(p, each, -turns) + p * each_rest;
    double left = (turns - rint(turns)) + rest;
    left -= rint(left);
    const double quarters = rint(4.0 * left);
    const float x = (float)fma(-0.25, quarters, left), t = x * x;
    // (coefficients: (2 pi)^k / k!, of alternating sign)
    const float s = x * fmaf(t, fmaf(t, fmaf(t, fmaf(t, 42.0586939f, -76.7058563f), 81.6052475f), -41.3417015f), 6.28318548f);
    const float c = fmaf(t, fmaf(t, fmaf(t, fmaf(t, fmaf(t, -26.4262562f, 60.2446404f), -85.4568176f), 64.9393921f), -19.7392082f), 1.0f);
    const int quarter = (int)quarters & 3;
    sin = quarter & 1 ? c : s;
    cos = quarter & 1 ? s : c;
    if (quarter & 2) sin = -sin;
    if (quarter == 1 || quarter == 2) cos = -cos;
}
__device__ __forceinline__ void set_tokens(Tokens& t, const RotaryArgs& a, const RotarySegment& s, int first, int n, bool backward) {
    if ((int)threadIdx.x < n) {
        const int token = first + threadIdx.x, text = token / a.length, i = token - text * a.length;
        const bool counts = i < valid_length(a.lens, text, a.length);
        const int64_t place = (int64_t)i + (a.starts ? a.starts[text] : 0), at = s.placed ? place : i;
        const bool there = counts && (!s.placed || (place >= 0 && place < a.cache));
        t.position[threadIdx.x] = a.positions && counts ? a.positions[(int64_t)text * a.length + i] : place;
        t.x[threadIdx.x] = there ? text * s.x.batch + i * s.x.position : -1;
        t.y[threadIdx.x] = there ? text * s.y.batch + at * s.y.position : -1;
        if (backward) t.out[threadIdx.x] = text * s.out.batch + i * s.out.position;
    }
    __syncthreads();
    const int pairs = a.rotated / 2;
    for (int k = threadIdx.x; k < n * pairs; k += kRotaryThreads) {
        const int token = k / pairs, pair = k - token * pairs;
        sine_and_cosine(t.position[token], a.frequencies[pair], t.sin[token][pair], t.cos[token][pair]);
    }
    __syncthreads();
}
__device__ __forceinline__ void angles_of(const Tokens& t, int token, const Place& at, f32x4& cos, f32x4& sin) {
    cos = f32x4{1.0f, 1.0f, 1.0f, 1.0f}; sin = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    if (at.pair >= 0) { cos = *reinterpret_cast<const f32x4*>(&t.cos[token][at.pair]); sin = *reinterpret_cast<const f32x4*>(&t.sin[token][at.pair]); }
}
// A number that is the same in all lanes, in scalar registers
__device__ __forceinline__ int64_t uniform(int64_t x) {
    return (int64_t)((uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)(x >> 32)) << 32 | (uint32_t)__builtin_amdgcn_readfirstlane((int)x));
}
// The first of some heads of a token
template <typename D> __device__ __forceinline__ uint8_t* heads_at(const Strided& s, int64_t token, int head) {
    return global_pointer(static_cast<uint8_t*>(const_cast<void*>(s.p)) + (token + head * s.head) * D::size);
}
// What a wave does one after another: heads of tokens
struct Walk {
    int token, block;                                                    // of the workgroup's tokens; of a token's heads
    __device__ __forceinline__ Walk(int u, int blocks) { token = u / blocks; block = u - token * blocks; }
    __device__ __forceinline__ void advance(int by_tokens, int by_blocks, int blocks) {
        token += by_tokens; block += by_blocks;
        if (block >= blocks) { block -= blocks; ++token; }
    }
};
__device__ __forceinline__ const RotarySegment& segment_of(const RotaryArgs& a, int& block, int& which) {
    which = 0;
    if (a.segments > 1 && block >= a.segment[1].first) which = 1;
    if (a.segments > 2 && block >= a.segment[2].first) which = 2;
    block -= a.segment[which].first;
    return a.segment[which];
}

template <int NORM, int GROUP> __device__ __forceinline__ void norm_head(Eight& x, float& factor, bool there, int head_dim, float eps) {
    factor = 1.0f;
    if constexpr (NORM != LSP_NORM_NONE) {
        const float share = 1.0f / (float)head_dim;
        if constexpr (NORM == LSP_NORM_LAYER) {
            float sum = 0.0f;
#pragma unroll
            for (int e = 0; e < 8; ++e) sum += x.x[e];
            const float mean = group_sum<GROUP>(sum) * share;
#pragma unroll
            for (int e = 0; e < 8; ++e) x.x[e] = there ? x.x[e] - mean : 0.0f;
        }
        float squares = 0.0f;
#pragma unroll
        for (int e = 0; e < 8; ++e) squares = fmaf(x.x[e], x.x[e], squares);
        // (v_rsq_f32, within an ulp, takes what is below 2^-126 for zero: where eps does not keep the sum above that, the root and quotient that IEEE has)
        const float sum = fmaf(group_sum<GROUP>(squares), share, eps);
        factor = eps >= 0x1p-126f ? __builtin_amdgcn_rsqf(sum) : 1.0f / sqrtf(sum);
        if (!there) factor = 0.0f;                                       // (of no head: one over the root of eps may be anything)
#pragma unroll
        for (int e = 0; e < 8; ++e) x.x[e] *= factor;
    }
}

// 4 x 1024 tokens of 32 + 32 heads of 128 in bf16, 134 MB: 24.4 us, 5.5 TB/s; 16384 tokens of 16 + 16 heads of 64 in fp32, 268 MB, 47.1 us, 5.7 TB/s.
template <typename D, int NORM, int GROUP, bool NEIGHBOURS>
__global__ __launch_bounds__(kRotaryThreads) void k_rotary(RotaryArgs a) {
    constexpr int kHeads = 64 / GROUP, kWaves = kRotaryThreads / 64;     // heads that a wave has at a time
    __shared__ Tokens t;
    int block = blockIdx.x, which;
    const RotarySegment& s = segment_of(a, block, which);
    const int group = block / s.parts, part = block - group * s.parts, first = group * s.tokens, n = min(s.tokens, a.batch * a.length - first);
    const Place at(a, threadIdx.x % GROUP);
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), own = (threadIdx.x & 63) / GROUP;
    const int blocks = (s.heads + kHeads - 1) / kHeads, step = kWaves * s.parts, by_tokens = step / blocks, by_blocks = step - by_tokens * blocks;
    const Eight w = load_vector<D>(which < 2 ? s.weight : nullptr, at, 1.0f), bias = load_vector<D>(which < 2 ? s.bias : nullptr, at, 0.0f);
    const Reach from = reach_of<D>(at, s.x, own), to = reach_of<D>(at, s.y, own);
    set_tokens(t, a, s, first, n, false);
    Walk now(part * kWaves + wave, blocks);
    const auto there = [&](const Walk& k) { return at.there && k.block * kHeads + own < s.heads; };
    const auto fetch = [&](const Walk& k) {
        Raw<D> r;
        r.a = r.b = u32x4{0, 0, 0, 0};
        if (k.token < n) {
            const int64_t x = uniform(t.x[k.token]);
            if (x >= 0 && there(k)) r = load_raw<D>(heads_at<D>(s.x, x, k.block * kHeads), from);
        }
        return r;
    };
    const auto work = [&](const Raw<D>& raw) {
        const int64_t y = uniform(t.y[now.token]);
        if (y < 0) return;                                               // (the token does not count, or its place is not in the cache)
        Eight x = widen_raw<D>(raw);
        if (which < 2) {
            float factor;
            norm_head<NORM, GROUP>(x, factor, there(now), a.head_dim, a.eps);
            if constexpr (NORM != LSP_NORM_NONE) {
#pragma unroll
                for (int e = 0; e < 8; ++e) x.x[e] = fmaf(x.x[e], w.x[e], bias.x[e]);
            }
            f32x4 cos, sin;
            angles_of(t, now.token, at, cos, sin);
            turn<NEIGHBOURS, false>(x, cos, sin);
        }
        if (there(now)) store_raw<D>(heads_at<D>(s.y, y, now.block * kHeads), to, x);
    };
    // two sets of registers, one asked for while the other is worked on
    Raw<D> even = fetch(now), odd;
    while (now.token < n) {
        Walk next = now;
        next.advance(by_tokens, by_blocks, blocks);
        odd = fetch(next);
        work(even);
        now = next;
        if (now.token >= n) break;
        next.advance(by_tokens, by_blocks, blocks);
        even = fetch(next);
        work(odd);
        now = next;
    }
}

// With y = xhat w + b turned by the angle, and d the gradient of the result turned back:  dw += d xhat, db += d, and with e = d w
//   dx = factor (e - xhat mean(e xhat) [- mean(e), for a norm with means]).
// Five waves a SIMD in 16 bits, for which sums of biases are left out where nobody asks for them (BIAS): 3 x 777 padded tokens of 16 + 4 heads of 80 in fp16, with means and biases, 12.0 us, with four
// waves 15.6; 4 x 1024 tokens of 32 + 32 heads of 128 in bf16, 38.9 us (5.2 TB/s), with four 42.1.
template <typename D, int NORM, int GROUP, bool NEIGHBOURS, bool BIAS>
__global__ __launch_bounds__(kRotaryThreads, D::size == 4 ? 4 : 5) void k_rotary_back(RotaryArgs a) {
    constexpr int kHeads = 64 / GROUP, kWaves = kRotaryThreads / 64, kGroups = kRotaryThreads / GROUP;
    __shared__ Tokens t;
    int block = blockIdx.x, which;
    const RotarySegment& s = segment_of(a, block, which);
    const Place at(a, threadIdx.x % GROUP);
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), own = (threadIdx.x & 63) / GROUP;
    const int blocks = (s.heads + kHeads - 1) / kHeads, step = kWaves * s.parts, by_tokens = step / blocks, by_blocks = step - by_tokens * blocks;
    const int tokens = a.batch * a.length, groups = (tokens + s.tokens - 1) / s.tokens * s.parts;
    const Eight w = load_vector<D>(s.weight, at, 1.0f);
    const Reach of_x = reach_of<D>(at, s.x, own), of_d = reach_of<D>(at, s.y, own), of_out = reach_of<D>(at, s.out, own);
    Eight dw, db;
#pragma unroll
    for (int e = 0; e < 8; ++e) dw.x[e] = db.x[e] = 0.0f;
    struct Both { Raw<D> d, x; };
    for (; block < groups; block += s.blocks) {
        const int group = block / s.parts, part = block - group * s.parts, first = group * s.tokens, n = min(s.tokens, tokens - first);
        __syncthreads();                                                 // (the tokens before are done with)
        set_tokens(t, a, s, first, n, true);
        Walk now(part * kWaves + wave, blocks);
        const auto there = [&](const Walk& k) { return at.there && k.block * kHeads + own < s.heads; };
        const auto fetch = [&](const Walk& k) {
            Both r;
            r.d.a = r.d.b = r.x.a = r.x.b = u32x4{0, 0, 0, 0};
            if (k.token < n) {
                const int64_t y = uniform(t.y[k.token]), x = uniform(t.x[k.token]);
                if (y >= 0 && there(k)) {
                    r.d = load_raw<D>(heads_at<D>(s.y, y, k.block * kHeads), of_d);
                    if constexpr (NORM != LSP_NORM_NONE) r.x = load_raw<D>(heads_at<D>(s.x, x, k.block * kHeads), of_x);
                }
            }
            return r;
        };
        const auto work = [&](const Both& raw) {
            Eight d = widen_raw<D>(raw.d);
            if (uniform(t.y[now.token]) >= 0) {                          // (otherwise d is zeros, and stays)
                f32x4 cos, sin;
                angles_of(t, now.token, at, cos, sin);
                turn<NEIGHBOURS, true>(d, cos, sin);
                if constexpr (NORM != LSP_NORM_NONE) {
                    Eight x = widen_raw<D>(raw.x);
                    float factor;
                    norm_head<NORM, GROUP>(x, factor, there(now), a.head_dim, a.eps);
                    float along = 0.0f, sum = 0.0f;
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        dw.x[e] = fmaf(d.x[e], x.x[e], dw.x[e]);
                        if constexpr (BIAS) db.x[e] += d.x[e];
                        d.x[e] *= w.x[e];
                        along = fmaf(d.x[e], x.x[e], along);
                        sum += d.x[e];
                    }
                    const float share = 1.0f / (float)a.head_dim;
                    along = group_sum<GROUP>(along) * share;
                    const float mean = NORM == LSP_NORM_LAYER ? group_sum<GROUP>(sum) * share : 0.0f;
#pragma unroll
                    for (int e = 0; e < 8; ++e) d.x[e] = factor * (d.x[e] - fmaf(x.x[e], along, mean));
                }
            }
            if (there(now)) store_raw<D>(heads_at<D>(s.out, uniform(t.out[now.token]), now.block * kHeads), of_out, d);
        };
        Both even = fetch(now), odd;
        while (now.token < n) {
            Walk next = now;
            next.advance(by_tokens, by_blocks, blocks);
            odd = fetch(next);
            work(even);
            now = next;
            if (now.token >= n) break;
            next.advance(by_tokens, by_blocks, blocks);
            even = fetch(next);
            work(odd);
            now = next;
        }
    }
    if (NORM == LSP_NORM_NONE || !a.sums) return;
    __shared__ float all[kGroups][GROUP * 8 + 4];
#pragma unroll
    for (int k = 0; k < (BIAS ? 2 : 1); ++k) {
        __syncthreads();
        if (at.there) {
#pragma unroll
            for (int e = 0; e < 8; ++e) all[threadIdx.x / GROUP][e < 4 ? at.first + e : at.second + e - 4] = k ? db.x[e] : dw.x[e];
        }
        __syncthreads();
        if ((int)threadIdx.x < a.head_dim) {
            float x = 0.0f;
#pragma unroll
            for (int g = 0; g < kGroups; ++g) x += all[g][threadIdx.x];
            a.partial[((int64_t)blockIdx.x * 2 + k) * a.head_dim + threadIdx.x] = x;
        }
    }
}

// The workgroups' parts of a sum, added in their order: 16 columns of one sum a workgroup, 64 runs of parts side by side.  (640 parts of 128 columns: 4.5 us, a launch and two reads.)
__global__ __launch_bounds__(1024) void k_rotary_sums(RotaryArgs a) {
    const RotarySegment& s = a.segment[blockIdx.y >> 1];
    const int k = blockIdx.y & 1, column = blockIdx.x * 16 + (threadIdx.x & 15), run = threadIdx.x >> 4;
    float* const to = k ? s.bias_sum : s.weight_sum;
    if (!to) return;                                                     // (and if nobody asks for a bias' sum there is none)
    float x = 0.0f;
    if (column < a.head_dim) {
#pragma unroll 8
        for (int p = run; p < s.blocks; p += 64) x += a.partial[((int64_t)(s.first + p) * 2 + k) * a.head_dim + column];
    }
    __shared__ float all[64][17];
    all[run][threadIdx.x & 15] = x;
    __syncthreads();
    if (run == 0 && column < a.head_dim) {
        float sum = 0.0f;
#pragma unroll 16
        for (int r = 0; r < 64; ++r) sum += all[r][threadIdx.x & 15];
        to[column] = sum;
    }
}

static int group_of(int head_dim) { return head_dim <= 32 ? 4 : head_dim <= 64 ? 8 : 16; }

// A workgroup has the tokens whose heads give each of its waves 16 steps, or as few as give 1024 workgroups; where one token each gives fewer, its heads are shared.
// Backward with sums: at most 640 workgroups of each that go on, as many as run at once, since each leaves a part of the sums.
void plan_rotary(RotaryArgs& a, bool backward) {
    const int64_t tokens = (int64_t)a.batch * a.length;
    const int at_a_time = 64 / group_of(a.head_dim), waves = kRotaryThreads / 64;
    a.blocks = 0;
    for (int k = 0; k < a.segments; ++k) {
        RotarySegment& s = a.segment[k];
        const int steps = (s.heads + at_a_time - 1) / at_a_time;          // of a token
        s.tokens = (int)std::min<int64_t>({std::max(1, 16 * waves / steps), kRotaryTokens, std::max<int64_t>(1, tokens / 1024)});
        const int64_t of_tokens = (tokens + s.tokens - 1) / s.tokens;
        s.parts = s.tokens > 1 ? 1 : (int)std::min<int64_t>((steps + waves - 1) / waves, std::max<int64_t>(1, 1024 / of_tokens));
        const int64_t blocks = of_tokens * s.parts;
        s.first = a.blocks;
        s.blocks = (int)(backward && a.sums ? std::min<int64_t>(blocks, 640) : blocks);
        a.blocks += s.blocks;
    }
}
size_t rotary_partial_bytes(const RotaryArgs& a) { return a.sums ? align_up((size_t)a.blocks * 2 * a.head_dim * sizeof(float), 256) : 0; }

template <typename D, int NORM, int GROUP> static void launch_one(const RotaryArgs& a, bool backward, hipStream_t st) {
    const dim3 grid((unsigned)a.blocks), block(kRotaryThreads);
    if (backward) {
        const bool bias = NORM != LSP_NORM_NONE && (a.segment[0].bias_sum || a.segment[1].bias_sum);
        const auto with = [&](auto b) {
            if (a.neighbours) hipLaunchKernelGGL((k_rotary_back<D, NORM, GROUP, true, decltype(b)::value>), grid, block, 0, st, a);
            else hipLaunchKernelGGL((k_rotary_back<D, NORM, GROUP, false, decltype(b)::value>), grid, block, 0, st, a);
        };
        if constexpr (NORM == LSP_NORM_NONE) with(std::false_type{});
        else if (bias) with(std::true_type{});
        else with(std::false_type{});
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
    hipLaunchKernelGGL(k_rotary_sums, dim3((unsigned)((a.head_dim + 15) / 16), 4), dim3(1024), 0, st, a);
    return hipGetLastError();
}

}  // namespace lsp

// The backward pass of attention.  The probabilities are made again from Q, K and the forward pass's L, tile by tile; no matrix of queries by
// keys is ever in memory.  With delta_i = dO_i . O_i:
//     P = exp(scale Q K^T - L),   dP = keep (dO V^T),   dS = P (dP - delta),
//     dV = (keep P)^T dO,   dQ = scale dS K,   dK = scale dS^T Q    (the last two summed over the query heads of a key head).
// Two kinds of workgroups in one launch, each owner of what it writes, so that nothing is added by atomics and the result does not depend on timing:
// attention_dq walks the keys for 128 queries, attention_dkv the queries for 128 keys, first in the launch, because theirs take longer.  Both make the scores, seven products
// instead of five; the other ways cost more memory than the two products take time (dS in memory, read again: 270 MB for four texts of 1024 with 32 heads, 52 us for two of
// seven products of 145; parts of dQ for every tile of keys in fp32: 600 MB).
//
// attention_dq has a query per lane, as the forward pass: S^T = K Q^T and dP^T = V dO^T give dS^T, the operand of dQ^T += K^T dS^T as it is.
// attention_dkv has a key per lane: S = Q K^T and dP = dO V^T (keys and values of the lane in registers) give the operands P and dS of
// dV^T += dO^T P and dK^T += Q^T dS; L and delta of the 16 queries of a lane come from LDS.
//
// fp16: gradients of scores can be far below what fp16 resolves, or above its range.  dP and delta are at most B = max |dO_i| max |V_j| keep, so
// with the power of two g <= 1 / B the operand 2^14 P g (dP - delta) neither overflows nor loses more than values 2^-38 of B; P itself is
// scaled by 2^14.  Powers of two change nothing else, and the sums are scaled back at the end.  bf16 and fp32 have the range of fp32.
//
// What is rounded to 16 bits: P and dS, as operands of the second products (the matrix cores take both operands in one type, and dS in two parts would be two products more of
// seven), and O, which delta is made of (its own fp32 values would be as much memory again as Q and dO).  With the results' own rounding dQ and dK are about 1.5 times as far from
// the exact ones as results rounded once: 0.0025 of their norm in bf16, 0.0003 in fp16.
//
// Bound by the matrix cores, at the clock that they leave.  Four texts of 1024, 32 heads of 128, causal, bf16: 145 us, 120 GFLOP of seven products, 0.83 PFLOP/s (0.93 with what
// the diagonal tiles make in vain); one of 8192, 16 heads: 800 to 915 us, 962 GFLOP, 1.05 to 1.2 PFLOP/s (a product of 8192 x 8192 matrices reaches 1.24 to 1.28).
#pragma once

#include <algorithm>

#include "attention_forward.h"

#if defined(__HIPCC__)
namespace lsp {

// The larger of two numbers, or the NaN if one is
__device__ __forceinline__ float larger(float x, float y) { return !(y <= x) ? y : x; }

template <typename D> constexpr float kLiftLog2 = std::is_same<D, F16>::value ? 14.0f : 0.0f;
template <typename D> constexpr float kLift = std::is_same<D, F16>::value ? 16384.0f : 1.0f;   // factor of the probabilities

// g: a power of two, at most 1 / (the largest |dP|); 1 where that is no number
template <typename D> __device__ __forceinline__ float score_factor(const AttentionArgs& a, int lane) {
    if constexpr (!std::is_same<D, F16>::value) return 1.0f;
    float largest[2] = {0.0f, 0.0f};
    for (int i = 4 * lane; i < a.norm_slots; i += 256)
#pragma unroll
        for (int which = 0; which < 2; ++which) {
            const f32x4 v = *reinterpret_cast<const f32x4*>(a.norms + which * kNormSlots + i);
#pragma unroll
            for (int j = 0; j < 4; ++j) if (i + j < a.norm_slots) largest[which] = larger(largest[which], v[j]);
        }
#pragma unroll
    for (int s = 1; s < 64; s <<= 1)
#pragma unroll
        for (int which = 0; which < 2; ++which) largest[which] = larger(largest[which], __shfl_xor(largest[which], s));
    const float bound = sqrtf(largest[0]) * sqrtf(largest[1]) * a.drop.scale * 1.01f;
    if (!(bound > 0.0f) || !(bound < INFINITY)) return 1.0f;
    return __uint_as_float((uint32_t)min(max(254 - (int)(__float_as_uint(bound) >> 23) - 1, 1), 254) << 23);
}

// delta of every query that counts; fp16: the largest norms too, of rows of dO and of V.  Bound by memory: 67 MB of bf16 in 12.4 us, 5.4 TB/s.  16 lanes have a row, eight elements each; `blocks`: of 16 rows, of dO
// and then of V, that the workgroups go through.  (What the workgroups of fp16 find they leave side by side: an atomic that all of them wait for took longer than the rest.)
template <typename D>
__global__ __launch_bounds__(256) void k_attention_delta(const AttentionArgs a, int64_t o_blocks, int64_t blocks) {
    const int lane = threadIdx.x & 63, part = lane & 15, col = 8 * part;
    float largest[2] = {0.0f, 0.0f};
    for (int64_t block = blockIdx.x; block < blocks; block += gridDim.x) {
        const bool values = block >= o_blocks;
        const int len = values ? a.k_len : a.q_len, heads = values ? a.kv_heads : a.heads;
        const int64_t row = (values ? block - o_blocks : block) * 16 + (threadIdx.x >> 4);
        const bool there = row < (int64_t)a.batch * heads * len;
        const uint32_t line = there ? (uint32_t)row / (uint32_t)len : 0u;                 // (there are fewer than 2^27 rows)
        const int i = there ? (int)((uint32_t)row - line * (uint32_t)len) : 0, b = (int)(line / (uint32_t)heads), head = (int)(line - (uint32_t)(b * heads));
        const bool counts = there && i < valid_length(values ? a.k_lens : a.q_lens, b, len);
        float dot = 0.0f, norm = 0.0f;
        if (counts && col < a.head_dim) {
            const uint8_t* p = at<D>(values ? a.v : a.d_o, b, i, head) + col * D::size;
            const uint8_t* q = values ? p : at<D>(a.o, b, i, head) + col * D::size;
            typename D::elem x[8], y[8];
            __builtin_memcpy(x, __builtin_assume_aligned(p, 16), sizeof(x));
            __builtin_memcpy(y, __builtin_assume_aligned(q, 16), sizeof(y));
#pragma unroll
            for (int e = 0; e < 8; ++e) { const float u = widen<D>(x[e]); dot = fmaf(u, widen<D>(y[e]), dot); norm = fmaf(u, u, norm); }
        }
#pragma unroll
        for (int s = 1; s < 16; s <<= 1) { dot += __shfl_xor(dot, s); norm += __shfl_xor(norm, s); }
        if (!values && counts && part == 0) a.delta[row] = dot;
        if (values) largest[1] = larger(largest[1], norm);
        else largest[0] = larger(largest[0], norm);
    }
    if constexpr (std::is_same<D, F16>::value) {
        __shared__ float found[2][4];
#pragma unroll
        for (int which = 0; which < 2; ++which) {
#pragma unroll
            for (int s = 16; s < 64; s <<= 1) largest[which] = larger(largest[which], __shfl_xor(largest[which], s));
            if (lane == 0) found[which][threadIdx.x >> 6] = largest[which];
        }
        __syncthreads();
        if (threadIdx.x < 2) {
            const float* n = found[threadIdx.x];
            a.norms[threadIdx.x * kNormSlots + blockIdx.x] = larger(larger(n[0], n[1]), larger(n[2], n[3]));
        }
    }
}

// Where the parts of dQ begin: behind those of dK and dV
__host__ __device__ static inline float* query_partial(const AttentionArgs& a) {
    return a.partial + (a.key_parts > 1 ? (int64_t)2 * a.key_parts * a.batch * a.kv_heads * a.k_len * a.head_dim : 0);
}

template <typename D, int DP, bool DROP>
__device__ __forceinline__ void attention_dq(const AttentionArgs& a, uint32_t block, uint8_t* smem) {
    using T = Tile<D, DP>;
    constexpr int kRows = kBackwardRows;
    constexpr int BN = tile_rows<D>(), NT = 256, kSteps = DP / 16, kTiles = BN / 32, kCols = DP / 32;
    constexpr uint32_t kTileBytes = BN * T::kRowBytes;
    const Lds lds = (Lds)smem;                                                            // K | V, twice
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), h = lane >> 5;
    int unit, tile;
    const int tiles = (a.q_len + kRows - 1) / kRows;
    work_of_block(block, (uint32_t)a.batch * a.heads * a.query_parts, tiles, unit, tile);
    const int row_tile = tiles - 1 - tile;
    const int part = unit % a.query_parts, head = unit / a.query_parts % a.heads, b = unit / a.query_parts / a.heads, kv_head = head / a.group;
    const int nq = valid_length(a.q_lens, b, a.q_len), nk = valid_length(a.k_lens, b, a.k_len), ahead = nk - nq;

    const int first = row_tile * kRows + wave * 32, qi = first + (lane & 31);
    const bool counts = qi < nq;
    const int limit = counts ? (a.causal ? min(nk, qi + ahead + 1) : nk) : 0;
    const int last_row = min(row_tile * kRows + kRows, nq) - 1;
    const int end_all = row_tile * kRows >= nq ? 0 : max(0, a.causal ? min(nk, last_row + ahead + 1) : nk);
    const int tiles_k = (end_all + BN - 1) / BN;                                          // of which this part has an equal share
    const int begin = tiles_k * part / a.query_parts * BN, end = min(end_all, tiles_k * (part + 1) / a.query_parts * BN);
    const int most = first >= nq ? 0 : a.causal ? min(nk, min(first + 31, nq - 1) + ahead + 1) : nk;
    const int least = first + 31 >= nq ? 0 : a.causal ? min(nk, first + ahead + 1) : nk;

    const float factor = score_factor<D>(a, lane), keep = (DROP ? a.drop.scale : 1.0f) * factor;
    float shift = 0.0f, delta = 0.0f;
    if (counts) {
        const int64_t line = ((int64_t)b * a.heads + head) * a.q_len + qi;
        const float L = a.L[line];
        shift = L == -INFINITY ? 0.0f : kLiftLog2<D> - L * 1.44269504f;
        delta = a.delta[line] * factor;
    }
    const float c2 = a.scale_log2;
    f32x16 dq[kCols];
#pragma unroll
    for (int c = 0; c < kCols; ++c) dq[c] = zeros16();

    const uint8_t* kp = at<D>(a.k, b, 0, kv_head);
    const uint8_t* vp = at<D>(a.v, b, 0, kv_head);
    const int64_t k_bytes = a.k.position * D::size, v_bytes = a.v.position * D::size;
    Fetch<D, DP, BN, NT> fetch_k, fetch_v;
    fetch_k.setup((uint32_t)k_bytes, a.head_dim, wave, lane);
    fetch_v.setup((uint32_t)v_bytes, a.head_dim, wave, lane);
    const Reader<D, DP> read(lane);
    if (begin < end) {
        Frag<D> qf[kSteps], gf[kSteps];
        if constexpr (D::size == 4) {
            const uint8_t* p = counts ? at<D>(a.q, b, qi, head) : nullptr;
            const uint8_t* g = counts ? at<D>(a.d_o, b, qi, head) : nullptr;
#pragma unroll
            for (int ks = 0; ks < kSteps; ++ks) { qf[ks] = global_frag(p, ks, a.head_dim, lane); gf[ks] = global_frag(g, ks, a.head_dim, lane); }
        } else {
            // the wave's queries and their gradients come through the buffers, each through half of them
            const Lds rows = lds + wave * 32 * T::kRowBytes, others = rows + kRows * T::kRowBytes;
            const auto fetch_rows = [&](const Strided& from, Lds to) {
                const uint32_t row_bytes = (uint32_t)(from.position * D::size);
                fetch_wave_rows<D, DP>(buffer_from(at<D>(from, b, first, head)), to, a.head_dim, lane, [&](uint32_t r) { return first + (int)r < nq ? r * row_bytes : kNowhere; });
            };
            fetch_rows(a.q, rows);
            fetch_rows(a.d_o, others);
            __builtin_amdgcn_s_waitcnt(0x0F70);
#pragma unroll
            for (int ks = 0; ks < kSteps; ++ks) { qf[ks] = read.rows(rows, 0, ks); gf[ks] = read.rows(others, 0, ks); }
            __syncthreads();
        }
        fetch_k(kp + begin * k_bytes, nk - begin, lds, wave);
        fetch_v(vp + begin * v_bytes, nk - begin, lds + kTileBytes, wave);
        arrived_for_all();
        const auto step = [&](Lds __restrict buf, Lds __restrict other, int k0) {
            if (k0 + BN < end) {
                fetch_k(kp + (k0 + BN) * k_bytes, nk - k0 - BN, other, wave);
                fetch_v(vp + (k0 + BN) * v_bytes, nk - k0 - BN, other + kTileBytes, wave);
            }
            if (k0 < most) {
                const bool edge = k0 + BN > least;
                const int seen = limit - k0 - 4 * h;
#pragma unroll
                for (int t = 0; t < kTiles; ++t) {
                    f32x16 s = zeros16(), dp = zeros16();
#pragma unroll
                    for (int ks = 0; ks < kSteps; ++ks) s = mma<D>(read.rows(buf, 32 * t, ks), qf[ks], s);
#pragma unroll
                    for (int ks = 0; ks < kSteps; ++ks) dp = mma<D>(read.rows(buf + kTileBytes, 32 * t, ks), gf[ks], dp);
                    Frag<D> kc[2][kCols];
#pragma unroll
                    for (int c = 0; c < kCols; ++c) kc[0][c] = read.columns(buf, 32 * t, c);
                    if constexpr (D::size == 2) {                                         // reads stay six ahead of their products
                        then_reads<6>();
#pragma unroll
                        for (int i = 0; i < 2 * kSteps - 6; ++i) { then_matrix<1>(); then_reads<1>(); }
                        then_matrix<6>();
                    }
                    if (edge)
#pragma unroll
                        for (int i = 0; i < 16; ++i) s[i] = 32 * t + 8 * (i >> 2) + (i & 3) < seen ? s[i] : -INFINITY;
                    const auto gradients = [&](int x) {                                   // of the scores of 16 keys
                        if constexpr (DROP) drop_keys(dp, x, k0 + 32 * t, qi, b * a.heads + head, a.drop, h);
#pragma unroll
                        for (int i = 8 * x; i < 8 * x + 8; ++i) s[i] = __builtin_amdgcn_exp2f(fmaf(s[i], c2, shift)) * fmaf(dp[i], keep, -delta);
                        return to_frag<D>(s, x);
                    };
                    // the other 16 keys' columns are read, and their gradients made, under the products of these
                    const Frag<D> ds0 = gradients(0);
                    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                    for (int c = 0; c < kCols; ++c) kc[1][c] = read.columns(buf, 32 * t + 16, c);
                    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                    for (int c = 0; c < kCols; ++c) dq[c] = mma<D>(kc[0][c], ds0, dq[c]);
                    const Frag<D> ds1 = gradients(1);
                    if constexpr (D::size == 2)
#pragma unroll
                        for (int c = 0; c < kCols; ++c) { then_matrix<1>(); then_vector<36 / kCols>(); }
                    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                    for (int c = 0; c < kCols; ++c) dq[c] = mma<D>(kc[1][c], ds1, dq[c]);
                }
            }
            arrived_for_all();
        };
        for (int k0 = begin; k0 < end; k0 += 2 * BN) {
            step(lds, lds + 2 * kTileBytes, k0);
            if (k0 + BN < end) step(lds + 2 * kTileBytes, lds, k0 + BN);
        }
    }
    const float back = a.scale / (factor * kLift<D>);
    if (a.query_parts > 1) {
        if (qi >= a.q_len) return;
        const int64_t lines = (int64_t)a.batch * a.heads * a.q_len, line = ((int64_t)b * a.heads + head) * a.q_len + qi;
        float* sums = query_partial(a) + (part * lines + line) * a.head_dim;
#pragma unroll
        for (int c = 0; c < kCols; ++c)
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                const int col = 32 * c + 8 * g + 4 * h;
                if (col < a.head_dim) *reinterpret_cast<f32x4*>(sums + col) = f32x4{dq[c][4 * g] * back, dq[c][4 * g + 1] * back, dq[c][4 * g + 2] * back, dq[c][4 * g + 3] * back};
            }
        return;
    }
    store_wave_rows<D, DP>(dq, back, lds + wave * 32 * T::kRowBytes, a.head_dim, lane,
                           [&](uint32_t r) -> uint8_t* { return first + (int)r < a.q_len ? const_cast<uint8_t*>(at<D>(a.dq, b, first + (int)r, head)) : nullptr; });
}

// Adds the parts of gradients, in order: `heads` x `len` rows of every batch each.  A thread has four columns, blockIdx.y is the gradient.  Bound by memory (90 MB of parts 16 us,
// 5.6 TB/s); where they are few, by its launch (4 us).
struct GradientParts { const float* from; Strided out; int32_t parts, heads, len; };
struct AddArgs { GradientParts g[3]; int32_t batch, head_dim; };
template <typename D>
__global__ __launch_bounds__(256) void k_attention_add(const AddArgs a) {
    const GradientParts& g = a.g[blockIdx.y];
    const int64_t lines = (int64_t)a.batch * g.heads * g.len;
    const int quads = a.head_dim / 4;
    const int64_t n = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (n >= lines * quads) return;
    const int64_t line = n / quads;
    const int col = (int)(n - line * quads) * 4;
    const float* from = g.from + line * a.head_dim + col;
    f32x4 sum = *reinterpret_cast<const f32x4*>(from);
    for (int p = 1; p < g.parts; ++p) sum += *reinterpret_cast<const f32x4*>(from + p * lines * a.head_dim);
    const int64_t head_line = line / g.len;
    const int i = (int)(line - head_line * g.len), b = (int)(head_line / g.heads), head = (int)(head_line - (int64_t)b * g.heads);
    store_four<D>(const_cast<uint8_t*>(at<D>(g.out, b, i, head)) + col * D::size, sum[0], sum[1], sum[2], sum[3]);
}

// At head_dim 128 in 16 bits K and V of a wave's keys, dK, dV and the scores are more than the 256 registers that two waves a SIMD have: V stays in
// LDS, and there is room for it with 32 queries at a time.
template <typename D, int DP> constexpr bool values_in_lds() { return D::size == 2 && DP > 96; }
template <typename D, int DP> constexpr int queries_at_once() { return values_in_lds<D, DP>() ? 32 : tile_rows<D>(); }

// LDS of attention_dkv: two buffers, where K (and V) come through before and the results go through after; the bits; V
template <typename D, int DP> constexpr uint32_t dkv_bits_at() {
    constexpr uint32_t row = Tile<D, DP>::kRowBytes, buffers = 2 * queries_at_once<D, DP>() * (2 * row + 8);
    constexpr uint32_t rows = kBackwardRows * row * (values_in_lds<D, DP>() || D::size == 4 ? 1 : 2);
    return buffers > rows ? buffers : rows;
}
template <typename D, int DP> constexpr uint32_t dkv_lds() {
    return dkv_bits_at<D, DP>() + 512 + (values_in_lds<D, DP>() ? kBackwardRows * Tile<D, DP>::kRowBytes : 0);
}
// and of attention_dq: two buffers, where Q and dO come through before
template <typename D, int DP> constexpr uint32_t dq_lds() {
    constexpr uint32_t tiles = 4 * tile_rows<D>(), rows = kBackwardRows * (D::size == 2 ? 2 : 1);
    return (tiles > rows ? tiles : rows) * Tile<D, DP>::kRowBytes;
}

template <typename D, int DP, bool DROP>
__device__ __forceinline__ void attention_dkv(const AttentionArgs& a, uint32_t block, uint8_t* smem) {
    using T = Tile<D, DP>;
    constexpr bool kValuesInLds = values_in_lds<D, DP>();
    constexpr int kKeys = kBackwardRows;
    constexpr int BQ = queries_at_once<D, DP>(), NT = 256, kSteps = DP / 16, kTiles = BQ / 32, kCols = DP / 32;
    constexpr uint32_t kTileBytes = BQ * T::kRowBytes, kBufBytes = 2 * kTileBytes + BQ * 8;
    constexpr uint32_t kBits = dkv_bits_at<D, DP>();                               // where the bits of dropout lie; V, if it stays, behind them
    const Lds lds = (Lds)smem;                                                            // Q | dO | L | delta, twice; bits of kept ones of each wave
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), h = lane >> 5;
    int unit, key_tile;                                                                   // (causal: the first keys have the most queries)
    work_of_block(block, (uint32_t)a.batch * a.kv_heads * a.key_parts, (a.k_len + kKeys - 1) / kKeys, unit, key_tile);
    const int part = unit % a.key_parts, kv_head = unit / a.key_parts % a.kv_heads, b = unit / a.key_parts / a.kv_heads;
    const int nq = valid_length(a.q_lens, b, a.q_len), nk = valid_length(a.k_lens, b, a.k_len), ahead = nk - nq;

    const int first = key_tile * kKeys + wave * 32, key = first + (lane & 31);
    const bool counts = key < nk;
    // queries from key - ahead on see the key; the workgroup's tiles begin at a multiple of BQ
    const int begin = a.causal ? max(0, key_tile * kKeys - ahead) / BQ * BQ : 0;
    const int end = key_tile * kKeys < nk ? nq : 0;
    const int from = a.causal ? max(0, first - ahead) : 0;                                // the wave's first query
    const int all_from = a.causal ? first + 31 - ahead : 0;                               // from here on every key of the wave is seen
    const int my_from = a.causal ? key - ahead : 0;

    const float factor = score_factor<D>(a, lane), keep = (DROP ? a.drop.scale : 1.0f) * factor, c2 = a.scale_log2;
    f32x16 dk[kCols], dv[kCols];
#pragma unroll
    for (int c = 0; c < kCols; ++c) { dk[c] = zeros16(); dv[c] = zeros16(); }

    const int64_t q_bytes = a.q.position * D::size, g_bytes = a.d_o.position * D::size;
    Fetch<D, DP, BQ, NT> fetch_q, fetch_g;
    fetch_q.setup((uint32_t)q_bytes, a.head_dim, wave, lane);
    fetch_g.setup((uint32_t)g_bytes, a.head_dim, wave, lane);
    float stat[2];                                                                        // threads below BQ: -L log2(e) and delta of a row
    const auto load = [&](int q_head, int q0, Lds buf) {
        fetch_q(at<D>(a.q, b, q0, q_head), nq - q0, buf, wave);
        fetch_g(at<D>(a.d_o, b, q0, q_head), nq - q0, buf + kTileBytes, wave);
        if (tid < BQ) {
            const int qi = q0 + tid;
            const int64_t line = ((int64_t)b * a.heads + q_head) * a.q_len + qi;
            const float L = qi < nq ? a.L[line] : -INFINITY;
            stat[0] = L == -INFINITY ? -INFINITY : kLiftLog2<D> - L * 1.44269504f;        // a row that sees nothing has probabilities 2^-inf
            stat[1] = L == -INFINITY ? 0.0f : a.delta[line] * factor;
        }
    };
    const auto store = [&](Lds buf) {
        if (tid < BQ) {
            lds_write<float>(buf + 2 * kTileBytes + tid * 4, stat[0]);
            lds_write<float>(buf + 2 * kTileBytes + BQ * 4 + tid * 4, stat[1]);
        }
    };
    // the steps are (query head of the group, tile of queries); this part has an equal share of them
    const int tiles_q = begin < end ? (end - begin + BQ - 1) / BQ : 0;
    const int step_from = (int)((int64_t)tiles_q * a.group * part / a.key_parts), step_past = (int)((int64_t)tiles_q * a.group * (part + 1) / a.key_parts);
    if (step_from < step_past) {
        const Reader<D, DP> read(lane);
        Frag<D> kf[kSteps], vf[kValuesInLds ? 1 : kSteps];
        const Lds rows = lds + wave * 32 * T::kRowBytes;
        const Lds values = kValuesInLds ? rows + kBits + 512 : rows + kKeys * T::kRowBytes;
        if constexpr (D::size == 4) {
            const uint8_t* p = counts ? at<D>(a.k, b, key, kv_head) : nullptr;
            const uint8_t* v = counts ? at<D>(a.v, b, key, kv_head) : nullptr;
#pragma unroll
            for (int ks = 0; ks < kSteps; ++ks) { kf[ks] = global_frag(p, ks, a.head_dim, lane); vf[ks] = global_frag(v, ks, a.head_dim, lane); }
        } else {
            // keys and values of the wave come through the buffers (V stays where it came to, if it stays in LDS)
            const auto fetch_rows = [&](const Strided& from, Lds to) {
                const uint32_t row_bytes = (uint32_t)(from.position * D::size);
                fetch_wave_rows<D, DP>(buffer_from(at<D>(from, b, first, kv_head)), to, a.head_dim, lane, [&](uint32_t r) { return first + (int)r < nk ? r * row_bytes : kNowhere; });
            };
            fetch_rows(a.k, rows);
            fetch_rows(a.v, values);
            __builtin_amdgcn_s_waitcnt(0x0F70);
#pragma unroll
            for (int ks = 0; ks < kSteps; ++ks) {
                kf[ks] = read.rows(rows, 0, ks);
                if constexpr (!kValuesInLds) vf[ks] = read.rows(values, 0, ks);
            }
            __syncthreads();
        }
        int steps = step_past - step_from;
        int q_head = kv_head * a.group + step_from / tiles_q, q0 = begin + step_from % tiles_q * BQ;
        load(q_head, q0, lds);
        store(lds);
        arrived_for_all();
        const auto step = [&](Lds __restrict buf, Lds __restrict other) {
            int next_head = q_head, next_q0 = q0 + BQ;
            if (next_q0 >= end) { next_q0 = begin; ++next_head; }
            const bool more = --steps > 0;
            if (more) load(next_head, next_q0, other);
            if (q0 + BQ > from && first < nk) {
                const bool edge = q0 < all_from;
                const int hidden = my_from - q0 - 4 * h;
#pragma unroll 1
                for (int t = 0; t < kTiles; ++t) {
                    f32x16 s = zeros16(), dp = zeros16();
#pragma unroll
                    for (int ks = 0; ks < kSteps; ++ks) s = mma<D>(read.rows(buf, 32 * t, ks), kf[ks], s);
#pragma unroll
                    for (int ks = 0; ks < kSteps; ++ks) {
                        Frag<D> v;
                        if constexpr (kValuesInLds) v = read.rows(values, 0, ks);
                        else v = vf[ks];
                        dp = mma<D>(read.rows(buf + kTileBytes, 32 * t, ks), v, dp);
                    }
                    // columns of dO and of Q by turns, 16 queries each; each is read under the products of the one before
                    Frag<D> gc[kCols], qc[kCols];
#pragma unroll
                    for (int c = 0; c < kCols; ++c) gc[c] = read.columns(buf + kTileBytes, 32 * t, c);
                    if constexpr (D::size == 2) {                                         // reads stay six ahead of their products
                        then_reads<6>();
#pragma unroll
                        for (int i = 0; i < 2 * kSteps - 6; ++i) { then_matrix<1>(); then_reads<1>(); }
                        then_matrix<6>();
                    }
                    if (edge)
#pragma unroll
                        for (int i = 0; i < 16; ++i) s[i] = 32 * t + 8 * (i >> 2) + (i & 3) >= hidden ? s[i] : -INFINITY;
                    u32x4 kept = {0, 0, 0, 0};
                    if constexpr (DROP) {
                        // eight lanes share a block of eight keys: of the 16 queries that they all have, each lane makes two; the bits go round by LDS
                        const Lds bits = lds + kBits + wave * 128 + (lane >> 3) * 16;
#pragma unroll
                        for (int half = 0; half < 2; ++half) {
                            const int x = (lane & 7) + 8 * half;
                            const u32x4 w = philox((uint32_t)key >> 3, q0 + 32 * t + 8 * (x >> 2) + 4 * h + (x & 3), b * a.heads + q_head, a.drop.offset, a.drop.key0, a.drop.key1);
                            uint32_t byte = 0;
#pragma unroll
                            for (int e = 0; e < 8; ++e) byte |= (philox_word(w, e) < a.drop.limit ? 0u : 1u) << e;
                            lds_write<uint8_t>(bits + x, (uint8_t)byte);
                        }
                        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
                        __builtin_amdgcn_wave_barrier();
                        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
                        kept = lds_read<u32x4>(bits) >> (uint32_t)(lane & 7);
                        __builtin_amdgcn_wave_barrier();
                    }
                    const auto probabilities = [&](int x) {                               // of 16 queries
                        f32x16 pd;
#pragma unroll
                        for (int g = 2 * x; g < 2 * x + 2; ++g) {
                            const f32x4 L = lds_read<f32x4>(buf + 2 * kTileBytes + (32 * t + 8 * g + 4 * h) * 4);
#pragma unroll
                            for (int j = 0; j < 4; ++j) {
                                const int i = 4 * g + j;
                                s[i] = __builtin_amdgcn_exp2f(fmaf(s[i], c2, L[j]));
                                pd[i] = DROP && !(kept[g] >> (8 * j) & 1u) ? 0.0f : s[i];
                            }
                        }
                        return to_frag<D>(pd, x);
                    };
                    const auto gradients = [&](int x) {
#pragma unroll
                        for (int g = 2 * x; g < 2 * x + 2; ++g) {
                            const f32x4 delta = lds_read<f32x4>(buf + 2 * kTileBytes + BQ * 4 + (32 * t + 8 * g + 4 * h) * 4);
#pragma unroll
                            for (int j = 0; j < 4; ++j) {
                                const int i = 4 * g + j;
                                s[i] *= fmaf(DROP && !(kept[g] >> (8 * j) & 1u) ? 0.0f : dp[i], keep, -delta[j]);
                            }
                        }
                        return to_frag<D>(s, x);
                    };
                    Frag<D> p = probabilities(0);
#pragma unroll
                    for (int x = 0; x < 2; ++x) {
                        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                        for (int c = 0; c < kCols; ++c) qc[c] = read.columns(buf, 32 * t + 16 * x, c);
                        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                        for (int c = 0; c < kCols; ++c) dv[c] = mma<D>(gc[c], p, dv[c]);
                        const Frag<D> ds = gradients(x);
                        if constexpr (D::size == 2)
#pragma unroll
                            for (int c = 0; c < kCols; ++c) { then_matrix<1>(); then_vector<20 / kCols>(); }
                        __builtin_amdgcn_sched_barrier(0);
                        if (x == 0) {
#pragma unroll
                            for (int c = 0; c < kCols; ++c) gc[c] = read.columns(buf + kTileBytes, 32 * t + 16, c);
                            __builtin_amdgcn_sched_barrier(0);
                        }
#pragma unroll
                        for (int c = 0; c < kCols; ++c) dk[c] = mma<D>(qc[c], ds, dk[c]);
                        if (x == 0) {
                            p = probabilities(1);
                            if constexpr (D::size == 2)
#pragma unroll
                                for (int c = 0; c < kCols; ++c) { then_matrix<1>(); then_vector<20 / kCols>(); }
                        }
                    }
                }
            }
            if (more) store(other);
            arrived_for_all();
            q_head = next_head; q0 = next_q0;
        };
        while (steps > 0) {
            step(lds, lds + kBufBytes);
            if (steps > 0) step(lds + kBufBytes, lds);
        }
    }
    const float back_v = (DROP ? a.drop.scale : 1.0f) / kLift<D>, back_k = a.scale / (factor * kLift<D>);
    if (!counts)                                                                          // (its scores were those of a row of zeros)
#pragma unroll
        for (int c = 0; c < kCols; ++c) { dk[c] = zeros16(); dv[c] = zeros16(); }
    if (a.key_parts > 1) {
        if (key >= a.k_len) return;
        const int64_t lines = (int64_t)a.batch * a.kv_heads * a.k_len, line = ((int64_t)b * a.kv_heads + kv_head) * a.k_len + key;
        float* sums = a.partial + (part * lines + line) * a.head_dim;                     // of dK; those of dV follow
#pragma unroll
        for (int c = 0; c < kCols; ++c)
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                const int col = 32 * c + 8 * g + 4 * h;
                if (col >= a.head_dim) continue;
                *reinterpret_cast<f32x4*>(sums + col) = f32x4{dk[c][4 * g] * back_k, dk[c][4 * g + 1] * back_k, dk[c][4 * g + 2] * back_k, dk[c][4 * g + 3] * back_k};
                *reinterpret_cast<f32x4*>(sums + a.key_parts * lines * a.head_dim + col) = f32x4{dv[c][4 * g] * back_v, dv[c][4 * g + 1] * back_v, dv[c][4 * g + 2] * back_v, dv[c][4 * g + 3] * back_v};
            }
        return;
    }
    const Lds room = lds + wave * 32 * T::kRowBytes;
    store_wave_rows<D, DP>(dk, back_k, room, a.head_dim, lane,
                           [&](uint32_t r) -> uint8_t* { return first + (int)r < a.k_len ? const_cast<uint8_t*>(at<D>(a.dk, b, first + (int)r, kv_head)) : nullptr; });
    __builtin_amdgcn_wave_barrier();
    store_wave_rows<D, DP>(dv, back_v, room, a.head_dim, lane,
                           [&](uint32_t r) -> uint8_t* { return first + (int)r < a.k_len ? const_cast<uint8_t*>(at<D>(a.dv, b, first + (int)r, kv_head)) : nullptr; });
}

// Both kinds in one launch, dK and dV first: neither waits for the other, and the last workgroups of the one leave no CU idle.  (In turns, with the longest of both
// kinds first, what is read is shared less: 178 instead of 150 us for four texts of 1024 with 32 heads of 128.)
template <typename D, int DP, bool DROP>
__global__ __launch_bounds__(256, (D::size == 4 && DP > 32 ? 1 : 2)) void k_attention_backward(const AttentionArgs a, uint32_t key_items) {
    extern __shared__ __align__(16) uint8_t smem[];
    if (blockIdx.x < key_items) attention_dkv<D, DP, DROP>(a, blockIdx.x, smem);
    else attention_dq<D, DP, DROP>(a, blockIdx.x - key_items, smem);
}

template <typename D, int DP, bool DROP> static hipError_t run_attention_backward(AttentionArgs a, hipStream_t st) {
    constexpr auto kern = k_attention_backward<D, DP, DROP>;
    constexpr int kRows = kBackwardRows;
    constexpr size_t lds = dkv_lds<D, DP>() > dq_lds<D, DP>() ? dkv_lds<D, DP>() : dq_lds<D, DP>();
    hipError_t e = allow_dynamic_lds<kern, lds>();
    if (e != hipSuccess) return e;
    const bool norms = std::is_same<D, F16>::value;
    const int64_t o_blocks = ((int64_t)a.batch * a.heads * a.q_len + 15) / 16;
    const int64_t blocks = o_blocks + (norms ? ((int64_t)a.batch * a.kv_heads * a.k_len + 15) / 16 : 0);
    const int64_t grid = norms ? std::min<int64_t>(blocks, kNormSlots) : blocks;
    a.norm_slots = (int32_t)grid;
    hipLaunchKernelGGL(k_attention_delta<D>, dim3((unsigned)grid), dim3(256), 0, st, a, o_blocks, blocks);
    if ((e = hipGetLastError()) != hipSuccess) return e;
    const int64_t key_items = (int64_t)a.batch * a.kv_heads * ((a.k_len + kRows - 1) / kRows) * a.key_parts;
    const int64_t query_items = (int64_t)a.batch * a.heads * ((a.q_len + kRows - 1) / kRows) * a.query_parts;
    hipLaunchKernelGGL(kern, dim3((unsigned)(key_items + query_items)), dim3(256), lds, st, a, (uint32_t)key_items);
    if ((e = hipGetLastError()) != hipSuccess) return e;
    AddArgs add{};
    add.batch = a.batch; add.head_dim = a.head_dim;
    int gradients = 0;
    int64_t rows = 0;
    const auto also = [&](const float* from, const Strided& out, int parts, int heads, int len) {
        add.g[gradients++] = {from, out, parts, heads, len};
        rows = std::max(rows, (int64_t)a.batch * heads * len);
    };
    if (a.key_parts > 1) {
        also(a.partial, a.dk, a.key_parts, a.kv_heads, a.k_len);
        also(a.partial + (int64_t)a.key_parts * a.batch * a.kv_heads * a.k_len * a.head_dim, a.dv, a.key_parts, a.kv_heads, a.k_len);
    }
    if (a.query_parts > 1) also(query_partial(a), a.dq, a.query_parts, a.heads, a.q_len);
    if (!gradients) return hipSuccess;
    hipLaunchKernelGGL(k_attention_add<D>, dim3((unsigned)((rows * (a.head_dim / 4) + 255) / 256), (unsigned)gradients), dim3(256), 0, st, add);
    return hipGetLastError();
}

template <typename D, int DP> static hipError_t run_attention_backward(const AttentionArgs& a, hipStream_t st) {
    return a.drop.limit ? run_attention_backward<D, DP, true>(a, st) : run_attention_backward<D, DP, false>(a, st);
}
template <typename D> hipError_t attention_backward_of(const AttentionArgs& a, hipStream_t st) {
    return a.head_dim <= 32 ? run_attention_backward<D, 32>(a, st) : a.head_dim <= 64 ? run_attention_backward<D, 64>(a, st)
         : a.head_dim <= 96 ? run_attention_backward<D, 96>(a, st) : run_attention_backward<D, 128>(a, st);
}

}  // namespace lsp
#endif

// The forward pass of attention: one pass over the keys with a running maximum and sum for each query.
//
// A workgroup has 128 or 256 query rows of a head, a wave 32 of them; tiles of keys and values go by in LDS, the next one on its way straight to its
// other half while the matrix cores work on the current.  The scores are made transposed, S^T = K Q^T: a lane then has all its scores (16 of every 32
// keys; lane l ^ 32 has the others) of ONE query, so maxima and sums stay in the lane, and the accumulators are the operand of
// O^T += V^T P^T as they are.
//
// The running maximum is moved only when a new one is larger by more than 2^8 (fp16: 2^4); until then probabilities are at most that much above its own, which
// neither their sum in fp32 nor their rounding minds, and the accumulators are left alone.  Probabilities are rounded to the storage type as operands of
// the second product, half a unit in the last place of each beside the result's own rounding (fp16: of those down to 2^-25 of the largest, see kTopLog2); their
// sums, and L, are made before that.
//
// Heads of 128: bound by the matrix cores (one text of 8192, 16 heads, causal, bf16: 255 to 300 us, 275 GFLOP, 0.9 to 1.1 PFLOP/s; four of 1024, 32 heads: 52 us, 34 GFLOP).
// Heads of 64: by exponentials and what else a score takes outside the matrix cores, a quarter-rate instruction and four others for 256 operations of theirs (16 heads, eight texts
// of 2048, fp16: 167 to 182 us, 137 GFLOP, 0.76 to 0.82 PFLOP/s; the vector units issue 70 % of the time, the matrix cores work 40 %).
#pragma once

#include "attention_few.h"

#if defined(__HIPCC__)
namespace lsp {

// Drops probabilities: registers i of `s` are keys key0 + 8 (i / 4) + 4 h + i % 4 of query q; those of `pair`, 8 of the 16.  A block of eight keys belongs to two
// lanes (h = 0, 1), four words each: of two blocks each lane makes one, and they swap the halves.
__device__ __forceinline__ void drop_keys(f32x16& s, int pair, uint32_t key0, uint32_t q, uint32_t head, const Dropout& drop, int h) {
    {
        const u32x4 w = philox((key0 >> 3) + 2 * pair + h, q, head, drop.offset, drop.key0, drop.key1);
        const auto a = __builtin_amdgcn_permlane32_swap(w[0], w[2], false, false);
        const auto b = __builtin_amdgcn_permlane32_swap(w[1], w[3], false, false);
#pragma unroll
        for (int x = 0; x < 2; ++x) {
            const uint32_t lo = a[x], hi = b[x];
            const int i = 8 * pair + 4 * x;
            s[i + 0] = (lo & 0xFFFFu) < drop.limit ? 0.0f : s[i + 0];
            s[i + 1] = (lo >> 16) < drop.limit ? 0.0f : s[i + 1];
            s[i + 2] = (hi & 0xFFFFu) < drop.limit ? 0.0f : s[i + 2];
            s[i + 3] = (hi >> 16) < drop.limit ? 0.0f : s[i + 3];
        }
    }
}

// Two waves a SIMD at heads of 128, three below: one waits or takes exponentials while the others multiply (eight texts of 2048, 16 heads of 64, fp16: 182 us, with two 188; heads of 96
// 236 and 242; 1073 queries and 2456 keys, heads of 32, 98 and 105; causal texts of 1024, heads of 64, 20 both, with four waves 27: all tiles at once, whatever their length).
template <typename D, int DP, bool DROP, int WAVES>
__global__ __launch_bounds__(64 * WAVES) __attribute__((amdgpu_waves_per_eu(2, DP <= 96 ? 3 : 2))) void k_attention_forward(const AttentionArgs a) {
    using T = Tile<D, DP>;
    constexpr int kRows = WAVES * kWaveRows;
    constexpr int BN = tile_rows<D>(), NT = 64 * WAVES, kSteps = DP / 16, kTiles = BN / 32, kCols = DP / 32;
    constexpr uint32_t kTileBytes = BN * T::kRowBytes;
    extern __shared__ __align__(16) uint8_t smem[];
    const Lds lds = (Lds)smem;                                                            // K | V, twice
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), h = lane >> 5;
    // which rows, of which head, and which part of the keys
    const int heads = a.packed ? a.kv_heads : a.heads;
    int unit, tile;
    // Where all workgroups run at once, two a CU, the longest goes with the shortest (causal, fp32, 2 texts of 1024, 16 heads of 128: 92 us, else 110; one of 943, heads of 64: 32 and 37;
    // 16 bits: even); else the longest come first.
    uint32_t block = blockIdx.x;
    if (WAVES == 4 && gridDim.x > 256 && gridDim.x <= 512 && gridDim.x % 8 == 0 && block >= 256)
        block = ((gridDim.x + 256) / 8 - 1 - block / 8) * 8 + block % 8;
    work_of_block(block, (uint32_t)a.batch * heads * a.splits, a.tiles, unit, tile);
    const int row_tile = a.tiles - 1 - tile;                                              // (causal: the longest first)
    const int split = unit % a.splits, head = unit / a.splits % heads, b = unit / a.splits / heads;
    const int kv_head = a.packed ? head : head / a.group;
    const int nq = valid_length(a.q_lens, b, a.q_len), nk = valid_length(a.k_lens, b, a.k_len);
    const int ahead = nk - nq;                                                            // query i sees keys up to i + ahead

    // this lane's row
    const int row = row_tile * kRows + wave * 32 + (lane & 31);
    const int q_head = a.packed ? kv_head * a.group + row / a.q_len : head;
    const int qi = a.packed ? row % a.q_len : row;
    const bool counts = row < a.rows && qi < nq;
    const int limit = counts ? (a.causal ? min(nk, qi + ahead + 1) : nk) : 0;             // it sees keys below
    // the keys of the workgroup: below the largest limit, in this split
    int most, least;                                                                      // of the wave
    if (a.packed || !a.causal) { most = nk; least = a.causal ? min(nk, ahead + 1) : nk; }
    else {
        const int first = row_tile * kRows + wave * 32;
        most = min(nk, min(first + 31, nq - 1) + ahead + 1);
        least = min(nk, first + ahead + 1);
    }
    const int last_row = min(row_tile * kRows + kRows, nq) - 1;
    const int end_all = a.packed || !a.causal ? nk : min(nk, last_row + ahead + 1);
    const int tiles_k = (max(end_all, 0) + BN - 1) / BN;                                  // of which this part has an equal share
    const int begin = tiles_k * split / a.splits * BN, end = min(end_all, tiles_k * (split + 1) / a.splits * BN);
    if (!a.packed && row_tile * kRows >= nq) most = 0;

    f32x16 o[kCols];
#pragma unroll
    for (int c = 0; c < kCols; ++c) o[c] = zeros16();
    float m = -INFINITY, l = 0.0f;                                                        // m: in the units of the scores; l: this lane's part
    const float c2 = a.scale_log2, slack = fminf(kLagLog2<D> / c2, 3e38f);    // (finite: the first maximum is above -infinity and it)

    const uint8_t* kp = at<D>(a.k, b, 0, kv_head);
    const uint8_t* vp = at<D>(a.v, b, 0, kv_head);
    const int64_t k_bytes = a.k.position * D::size, v_bytes = a.v.position * D::size;
    Fetch<D, DP, BN, NT> fetch_k, fetch_v;
    fetch_k.setup((uint32_t)k_bytes, a.head_dim, wave, lane);
    fetch_v.setup((uint32_t)v_bytes, a.head_dim, wave, lane);
    const bool any = begin < end && (a.packed || row_tile * kRows < nq);
    const Reader<D, DP> read(lane);
    const bool all_count = __all(counts);
    if (any) {
        Frag<D> qf[kSteps];
        if constexpr (D::size == 4) {
            const uint8_t* p = counts ? at<D>(a.q, b, qi, q_head) : nullptr;
#pragma unroll
            for (int ks = 0; ks < kSteps; ++ks) qf[ks] = global_frag(p, ks, a.head_dim, lane);
        }
        fetch_k(kp + begin * k_bytes, nk - begin, lds, wave);
        fetch_v(vp + begin * v_bytes, nk - begin, lds + kTileBytes, wave);
        if constexpr (D::size == 2) {
            // the wave's queries come through the second buffer while the first keys are on their way into the first
            const Lds rows = lds + 2 * kTileBytes + wave * 32 * T::kRowBytes;
            const int wave_row = row_tile * kRows + wave * 32;
            const uint32_t q_bytes = (uint32_t)(a.q.position * D::size);
            const Buffer q = buffer_from(at<D>(a.q, b, a.packed ? 0 : wave_row, a.packed ? kv_head * a.group : head));
            fetch_wave_rows<D, DP>(q, rows, a.head_dim, lane, [&](uint32_t r) {
                if (!a.packed) return wave_row + (int)r < nq ? r * q_bytes : kNowhere;
                const uint32_t n = wave_row + r, of_group = n / a.q_len, i = n - of_group * a.q_len;
                return (int)n < a.rows && (int)i < nq ? of_group * (uint32_t)(a.q.head * D::size) + i * q_bytes : kNowhere;
            });
            __builtin_amdgcn_s_waitcnt(0x0F70);
#pragma unroll
            for (int ks = 0; ks < kSteps; ++ks) qf[ks] = read.rows(rows, 0, ks);
        }
        arrived_for_all();
        const auto step = [&](Lds __restrict buf, Lds __restrict other, int k0) {
            if (k0 + BN < end) {
                fetch_k(kp + (k0 + BN) * k_bytes, nk - k0 - BN, other, wave);
                fetch_v(vp + (k0 + BN) * v_bytes, nk - k0 - BN, other + kTileBytes, wave);
            }
            if (k0 < most) {
                f32x16 s[kTiles];
#pragma unroll
                for (int t = 0; t < kTiles; ++t) {
                    s[t] = zeros16();
#pragma unroll
                    for (int ks = 0; ks < kSteps; ++ks) s[t] = mma<D>(read.rows(buf, 32 * t, ks), qf[ks], s[t]);
                }
                Frag<D> vf[2][kCols];
#pragma unroll
                for (int c = 0; c < kCols; ++c) vf[0][c] = read.columns(buf + kTileBytes, 0, c);
                if constexpr (D::size == 2) {                                             // reads stay six ahead of their products
                    then_reads<6>();
#pragma unroll
                    for (int i = 0; i < kTiles * kSteps - 6; ++i) { then_matrix<1>(); then_reads<1>(); }
                    then_matrix<6>();
                }
                if (k0 + BN > least || !all_count) {
                    const int seen = limit - k0 - 4 * h;
#pragma unroll
                    for (int t = 0; t < kTiles; ++t)
#pragma unroll
                        for (int i = 0; i < 16; ++i) s[t][i] = 32 * t + 8 * (i >> 2) + (i & 3) < seen ? s[t][i] : -INFINITY;
                }
                float top = s[0][0];
#pragma unroll
                for (int t = 0; t < kTiles; ++t)
#pragma unroll
                    for (int i = 0; i < 16; ++i) top = fmaxf(top, s[t][i]);
                top = halves_max(top);
                if (__any(top > m + slack)) {
                    const float m_new = fmaxf(m, top);
                    const float keep = m_new == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f((m - m_new) * c2);
                    m = m_new;
                    l *= keep;
#pragma unroll
                    for (int c = 0; c < kCols; ++c)
#pragma unroll
                        for (int i = 0; i < 16; ++i) o[c][i] *= keep;
                }
                const float shift = m == -INFINITY ? 0.0f : fmaf(-m, c2, kTopLog2<D>);
                const auto probabilities = [&](int x) {                                   // of keys 16 x .. 16 x + 15
                    f32x16& w = s[x >> 1];
                    float sum = 0.0f;
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        const int i = 8 * (x & 1) + j;
                        w[i] = __builtin_amdgcn_exp2f(fmaf(w[i], c2, shift));
                        sum += w[i];
                    }
                    l += sum;
                    if constexpr (DROP) drop_keys(w, x & 1, k0 + 32 * (x >> 1), qi, b * a.heads + q_head, a.drop, h);
                    return to_frag<D>(w, x & 1);
                };
                // the values of the next 16 keys are read, and their exponentials made, under the products of these
                Frag<D> p = probabilities(0);
#pragma unroll
                for (int x = 0; x < kTiles * 2; ++x) {
                    __builtin_amdgcn_sched_barrier(0);
                    Frag<D> next_p;
                    if (x + 1 < kTiles * 2) {
#pragma unroll
                        for (int c = 0; c < kCols; ++c) vf[(x + 1) & 1][c] = read.columns(buf + kTileBytes, 16 * (x + 1), c);
                        __builtin_amdgcn_sched_barrier(0);
                    }
#pragma unroll
                    for (int c = 0; c < kCols; ++c) o[c] = mma<D>(vf[x & 1][c], p, o[c]);
                    if (x + 1 < kTiles * 2) {
                        next_p = probabilities(x + 1);
                        if constexpr (D::size == 2) {
#pragma unroll
                            for (int c = 0; c < kCols; ++c) { then_matrix<1>(); then_vector<28 / kCols>(); }
                        }
                    }
                    p = next_p;
                }
                __builtin_amdgcn_sched_barrier(0);
            }
            arrived_for_all();
        };
        for (int k0 = begin; k0 < end; k0 += 2 * BN) {                                    // (by turns, so that the buffers are constants of the instructions)
            step(lds, lds + 2 * kTileBytes, k0);
            if (k0 + BN < end) step(lds + 2 * kTileBytes, lds, k0 + BN);
        }
    }
    l = halves_sum(l);
    if (a.splits > 1) {
        // this part's sums as they are; k_attention_join puts the parts together
        if (row >= a.rows) return;
        const int64_t lines = (int64_t)a.batch * a.heads * a.q_len;
        const int64_t line = ((int64_t)b * a.heads + q_head) * a.q_len + qi;
        float* out = a.partial + (split * lines + line) * a.head_dim;
#pragma unroll
        for (int c = 0; c < kCols; ++c)
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                const int col = 32 * c + 8 * g + 4 * h;
                if (col < a.head_dim) *reinterpret_cast<f32x4*>(out + col) = f32x4{o[c][4 * g], o[c][4 * g + 1], o[c][4 * g + 2], o[c][4 * g + 3]};
            }
        if (h == 0) *reinterpret_cast<f32x2*>(a.partial + a.splits * lines * a.head_dim + (split * lines + line) * 2) = f32x2{m, l};
        return;
    }
    const float inv = l == 0.0f ? 0.0f : (DROP ? a.drop.scale : 1.0f) / l;
    const int wave_row = row_tile * kRows + wave * 32;
    store_wave_rows<D, DP>(o, inv, lds + wave * 32 * T::kRowBytes, a.head_dim, lane, [&](uint32_t r) -> uint8_t* {
        const int n = wave_row + (int)r;
        if (n >= a.rows) return nullptr;
        return const_cast<uint8_t*>(a.packed ? at<D>(a.o, b, n % a.q_len, kv_head * a.group + n / a.q_len) : at<D>(a.o, b, n, head));
    });
    if (h == 0 && row < a.rows) a.L[((int64_t)b * a.heads + q_head) * a.q_len + qi] = l == 0.0f ? -INFINITY : m * a.scale + __logf(l * (1.0f / kTop<D>));
}

// Joins the parts of a row: O = sum_s w_s O_s / sum_s w_s l_s with w_s = 2^(m_s - m).  Bound by memory, and where parts are few by its launch (4 us).  A wave has a row: its lanes have a part's (m, l) each, and then two columns.
template <typename D>
__global__ __launch_bounds__(256) void k_attention_join(const AttentionArgs a) {
    const int64_t lines = (int64_t)a.batch * a.heads * a.q_len;
    const int64_t line = (int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if (line >= lines) return;
    const int lane = threadIdx.x & 63, col = 2 * lane;
    const f32x2* ml = reinterpret_cast<const f32x2*>(a.partial + a.splits * lines * a.head_dim);
    const f32x2 part = lane < a.splits ? ml[lane * lines + line] : f32x2{-INFINITY, 0.0f};       // (there are at most 64 parts)
    float m = part[0];
#pragma unroll
    for (int s = 1; s < 64; s <<= 1) m = fmaxf(m, __shfl_xor(m, s));
    const float w = part[0] == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f((part[0] - m) * a.scale_log2);
    float l = w * part[1], x = 0.0f, y = 0.0f;
#pragma unroll
    for (int s = 1; s < 64; s <<= 1) l += __shfl_xor(l, s);
    const float* o = a.partial + line * a.head_dim + min(col, a.head_dim - 2);
    for (int s = 0; s < a.splits; s += 4) {                                               // (a part past the last has no weight)
        f32x2 v[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) v[k] = *reinterpret_cast<const f32x2*>(o + min(s + k, a.splits - 1) * lines * a.head_dim);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const float f = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(w), min(s + k, 63)));
            x = s + k < a.splits ? fmaf(f, v[k][0], x) : x; y = s + k < a.splits ? fmaf(f, v[k][1], y) : y;
        }
    }
    const float inv = l == 0.0f ? 0.0f : a.drop.scale / l;
    const int64_t head_line = line / a.q_len;
    const int qi = (int)(line - head_line * a.q_len), b = (int)(head_line / a.heads), head = (int)(head_line - (int64_t)b * a.heads);
    if (col < a.head_dim) {
        typename D::elem* out = reinterpret_cast<typename D::elem*>(const_cast<uint8_t*>(at<D>(a.o, b, qi, head))) + col;
        out[0] = narrow<D>(x * inv); out[1] = narrow<D>(y * inv);
    }
    if (lane == 0) a.L[line] = l == 0.0f ? -INFINITY : m * a.scale + __logf(l * (1.0f / kTop<D>));
}

template <typename D> static hipError_t run_attention_join(const AttentionArgs& a, hipStream_t st) {
    const int64_t lines = (int64_t)a.batch * a.heads * a.q_len;
    hipLaunchKernelGGL(k_attention_join<D>, dim3((unsigned)((lines + 3) / 4)), dim3(256), 0, st, a);
    return hipGetLastError();
}

template <typename D, int DP, bool DROP, int WAVES> static hipError_t run_attention_forward(const AttentionArgs& a, hipStream_t st) {
    constexpr auto kern = k_attention_forward<D, DP, DROP, WAVES>;
    // two buffers of keys and values; the second is where the queries come through, and the results go through all of it
    constexpr size_t tiles = 4 * (size_t)tile_rows<D>(), rows = D::size == 2 ? tiles / 2 + WAVES * kWaveRows : WAVES * kWaveRows;
    constexpr size_t lds = (tiles > rows ? tiles : rows) * Tile<D, DP>::kRowBytes;
    hipError_t e = allow_dynamic_lds<kern, lds>();
    if (e != hipSuccess) return e;
    const int64_t items = (int64_t)a.batch * (a.packed ? a.kv_heads : a.heads) * a.tiles * a.splits;
    hipLaunchKernelGGL(kern, dim3((unsigned)items), dim3(64 * WAVES), lds, st, a);
    return hipGetLastError();
}

template <typename D, int DP, int WAVES> static hipError_t run_attention_forward(const AttentionArgs& a, hipStream_t st) {
    return a.drop.limit ? run_attention_forward<D, DP, true, WAVES>(a, st) : run_attention_forward<D, DP, false, WAVES>(a, st);
}
template <typename D, int WAVES> static hipError_t run_attention_forward(const AttentionArgs& a, hipStream_t st) {
    return a.head_dim <= 32 ? run_attention_forward<D, 32, WAVES>(a, st) : a.head_dim <= 64 ? run_attention_forward<D, 64, WAVES>(a, st)
         : a.head_dim <= 96 ? run_attention_forward<D, 96, WAVES>(a, st) : run_attention_forward<D, 128, WAVES>(a, st);
}
template <typename D> hipError_t attention_forward_of(const AttentionArgs& a, hipStream_t st) {
    hipError_t e;
    if constexpr (D::size == 2) e = a.few ? run_attention_few<D>(a, st)
                                  : a.waves == 8 ? (a.head_dim <= 96 ? run_attention_forward<D, 96, 8>(a, st) : run_attention_forward<D, 128, 8>(a, st))
                                                 : run_attention_forward<D, 4>(a, st);
    else e = run_attention_forward<D, 4>(a, st);
    return e != hipSuccess || a.splits == 1 ? e : run_attention_join<D>(a, st);
}

}  // namespace lsp
#endif

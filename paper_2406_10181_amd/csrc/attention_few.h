// The forward pass of attention for few queries (single tokens against a cache): at most 32 rows, all query heads of a key head together.
//
// Nothing but the keys and values matters here, each read once, and what bounds it is how much of them is on the way.  So the four waves of a workgroup go
// through keys of their own, 32 at a time, and wait for nobody: keys go straight into registers, one tile ahead, as the operands that they are (a lane has
// a row; a cycle a lane is less than memory takes), and values into LDS, one tile ahead, from where they are read transposed.  At the end the four waves' sums
// are joined in LDS, and those of several workgroups, if the keys of a head are split, by k_attention_join.
//
// 8 texts of up to 8192 keys, 32 heads over 8 key heads of 128, bf16, 185 MB: 35 to 39 us, 4.8 to 5.3 TB/s, and 5 for the join.  With half or twice as many parts 36.4 and 37.5 when
// this took 35.5; with loads that leave nothing in the caches 53; k_attention_forward, whose waves wait for one another at every tile, 39 and 8.
#pragma once

#include "attention.h"

#if defined(__HIPCC__)
namespace lsp {

constexpr int kFewKeys = 32;                                          // of a wave's step

template <typename D, int DP>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(2, 2))) void k_attention_few(const AttentionArgs a) {
    using T = Tile<D, DP>;
    constexpr int kSteps = DP / 16, kCols = DP / 32, kLine = DP * 4 + 16, kLoads = kSteps + T::kUnits / 2;
    constexpr uint32_t kTileBytes = kFewKeys * T::kRowBytes;
    extern __shared__ __align__(16) uint8_t smem[];
    const Lds lds = (Lds)smem;                                                            // two tiles of V for each wave; at the end sums
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), h = lane >> 5;
    const int heads = a.packed ? a.kv_heads : a.heads;
    int unit, tile;
    work_of_block(blockIdx.x, (uint32_t)a.batch * heads * a.splits, 1, unit, tile);
    const int split = unit % a.splits, head = unit / a.splits % heads, b = unit / a.splits / heads;
    const int kv_head = a.packed ? head : head / a.group;
    const int nq = valid_length(a.q_lens, b, a.q_len), nk = valid_length(a.k_lens, b, a.k_len), ahead = nk - nq;

    const int row = lane & 31, q_head = a.packed ? kv_head * a.group + row / a.q_len : head, qi = a.packed ? row % a.q_len : row;
    const bool counts = row < a.rows && qi < nq, all_count = __all(counts);
    const int limit = counts ? (a.causal ? min(nk, qi + ahead + 1) : nk) : 0, least = a.causal ? min(nk, ahead + 1) : nk;
    const int begin = split * a.split_tiles * kFewKeys, end = min(nk, begin + a.split_tiles * kFewKeys);

    Frag<D> qf[kSteps];
#pragma unroll
    for (int ks = 0; ks < kSteps; ++ks) {
        const int col = 16 * ks + 8 * h;
        qf[ks].w = u32x4{0, 0, 0, 0};
        if (counts && col < a.head_dim) qf[ks].w = *reinterpret_cast<const u32x4*>(at<D>(a.q, b, qi, q_head) + col * D::size);
    }
    f32x16 o[kCols];
#pragma unroll
    for (int c = 0; c < kCols; ++c) o[c] = zeros16();
    float m = -INFINITY, l = 0.0f;
    const float c2 = a.scale_log2, slack = fminf(kLagLog2<D> / c2, 3e38f);    // (finite: the first maximum is above -infinity and it)
    const Reader<D, DP> read(lane);
    const uint8_t* kp = at<D>(a.k, b, 0, kv_head);
    const uint8_t* vp = at<D>(a.v, b, 0, kv_head);
    const int64_t k_bytes = a.k.position * D::size, v_bytes = a.v.position * D::size;
    const auto fetch = [&](int k0, Frag<D> (&kf)[kSteps], Lds at) {
        const Buffer keys = buffer_from(kp + k0 * k_bytes), values = buffer_from(vp + k0 * v_bytes);
        const uint32_t off = k0 + row < end ? (uint32_t)row * (uint32_t)k_bytes + h * 16u : kNowhere;
#pragma unroll
        for (int ks = 0; ks < kSteps; ++ks) {
            const uint32_t o = 16 * ks + 8 * h < a.head_dim ? off + ks * 32u : kNowhere;
            kf[ks].w = __builtin_amdgcn_raw_buffer_load_b128(keys, (int)o, 0, 0);
        }
        fetch_wave_rows<D, DP>(values, at, a.head_dim, lane, [&](uint32_t r) { return k0 + (int)r < end ? r * (uint32_t)v_bytes : kNowhere; });
    };
    const Lds mine = lds + wave * 2 * kTileBytes;
    const int step_keys = 4 * kFewKeys;
    int k0 = begin + wave * kFewKeys;
    if (k0 < end) {
        Frag<D> ka[kSteps], kb[kSteps];
        const auto step = [&](Lds __restrict cur, Lds __restrict other, Frag<D> (&kf)[kSteps], Frag<D> (&next)[kSteps]) {
            fetch(k0 + step_keys, next, other);                                           // (past the end nothing is read: so many loads are on the way in every step)
            f32x16 s = zeros16();
#pragma unroll
            for (int ks = 0; ks < kSteps; ++ks) s = mma<D>(kf[ks], qf[ks], s);
            if (k0 + kFewKeys > least || k0 + kFewKeys > end || !all_count) {
                const int seen = min(limit, end) - k0 - 4 * h;
#pragma unroll
                for (int i = 0; i < 16; ++i) s[i] = 8 * (i >> 2) + (i & 3) < seen ? s[i] : -INFINITY;
            }
            float top = s[0];
#pragma unroll
            for (int i = 0; i < 16; ++i) top = fmaxf(top, s[i]);
            top = halves_max(top);
            if (__any(top > m + slack)) {
                const float m_new = fmaxf(m, top), keep = m_new == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f((m - m_new) * c2);
                m = m_new;
                l *= keep;
#pragma unroll
                for (int c = 0; c < kCols; ++c)
#pragma unroll
                    for (int i = 0; i < 16; ++i) o[c][i] *= keep;
            }
            const float shift = m == -INFINITY ? 0.0f : fmaf(-m, c2, kTopLog2<D>);
#pragma unroll
            for (int i = 0; i < 16; ++i) { s[i] = __builtin_amdgcn_exp2f(fmaf(s[i], c2, shift)); l += s[i]; }
            // the values of this step have arrived when no more is on the way than the next one's keys and values
            __builtin_amdgcn_s_waitcnt(0x0F70 | (kLoads & 15) | (kLoads >> 4) << 14);      // vmcnt(kLoads)
#pragma unroll
            for (int x = 0; x < 2; ++x) {
                const Frag<D> p = to_frag<D>(s, x);
#pragma unroll
                for (int c = 0; c < kCols; ++c) o[c] = mma<D>(read.columns(cur, 16 * x, c), p, o[c]);
            }
            k0 += step_keys;
        };
        fetch(k0, ka, mine);
        while (k0 < end) {
            step(mine, mine + kTileBytes, ka, kb);
            if (k0 < end) step(mine + kTileBytes, mine, kb, ka);
        }
    }
    l = halves_sum(l);
    // the four waves' sums: [wave][row] of O, then of (m, l)
    arrived_for_all();                                                                    // (the loads past the end write zeros)
    const Lds stats = lds + 4 * 32 * kLine;
#pragma unroll
    for (int c = 0; c < kCols; ++c)
#pragma unroll
        for (int g = 0; g < 4; ++g)
            lds_write<f32x4>(lds + (wave * 32 + row) * kLine + (32 * c + 8 * g + 4 * h) * 4, f32x4{o[c][4 * g], o[c][4 * g + 1], o[c][4 * g + 2], o[c][4 * g + 3]});
    if (h == 0) lds_write<f32x2>(stats + (wave * 32 + row) * 8, f32x2{m, l});
    __syncthreads();
    const int quads = a.head_dim / 4;
    const int64_t lines = (int64_t)a.batch * a.heads * a.q_len;
    for (int n = tid; n < a.rows * quads; n += 256) {
        const int r = n / quads, col = (n - r * quads) * 4;
        f32x2 ml[4];
        float top = -INFINITY, sum = 0.0f;
#pragma unroll
        for (int w = 0; w < 4; ++w) { ml[w] = lds_read<f32x2>(stats + (w * 32 + r) * 8); top = fmaxf(top, ml[w][0]); }
        f32x4 v = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            const float f = ml[w][0] == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f((ml[w][0] - top) * c2);
            sum += f * ml[w][1];
            v += f * lds_read<f32x4>(lds + (w * 32 + r) * kLine + col * 4);
        }
        const int rq_head = a.packed ? kv_head * a.group + r / a.q_len : head, ri = a.packed ? r % a.q_len : r;
        const int64_t line = ((int64_t)b * a.heads + rq_head) * a.q_len + ri;
        if (a.splits > 1) {
            *reinterpret_cast<f32x4*>(a.partial + (split * lines + line) * a.head_dim + col) = v;
            if (col == 0) *reinterpret_cast<f32x2*>(a.partial + a.splits * lines * a.head_dim + (split * lines + line) * 2) = f32x2{top, sum};
        } else {
            const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
            store_four<D>(const_cast<uint8_t*>(at<D>(a.o, b, ri, rq_head)) + col * D::size, v[0] * inv, v[1] * inv, v[2] * inv, v[3] * inv);
            if (col == 0) a.L[line] = sum == 0.0f ? -INFINITY : top * a.scale + __logf(sum * (1.0f / kTop<D>));
        }
    }
}

template <typename D, int DP> static hipError_t run_attention_few(const AttentionArgs& a, hipStream_t st) {
    constexpr auto kern = k_attention_few<D, DP>;
    constexpr size_t tiles = (size_t)8 * kFewKeys * Tile<D, DP>::kRowBytes, sums = (size_t)4 * 32 * (DP * 4 + 16 + 8), lds = tiles > sums ? tiles : sums;
    const hipError_t e = allow_dynamic_lds<kern, lds>();
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(kern, dim3((unsigned)(a.batch * (a.packed ? a.kv_heads : a.heads) * a.splits)), dim3(256), lds, st, a);
    return hipGetLastError();
}
template <typename D> static hipError_t run_attention_few(const AttentionArgs& a, hipStream_t st) {
    return a.head_dim <= 32 ? run_attention_few<D, 32>(a, st) : a.head_dim <= 64 ? run_attention_few<D, 64>(a, st)
         : a.head_dim <= 96 ? run_attention_few<D, 96>(a, st) : run_attention_few<D, 128>(a, st);
}

}  // namespace lsp
#endif

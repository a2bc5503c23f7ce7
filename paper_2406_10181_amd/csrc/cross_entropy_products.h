// The cross entropy's kernels with products in them, instantiated for each type in cross_entropy_{bf16,f16,f32}.hip.
#pragma once

#include "cross_entropy.h"
#include "matmul.h"

namespace lsp {

#if defined(__HIPCC__)
// 32 x 32: four groups of one wave each that share the length (64 tiles of length 4096 in bf16 9.7 us, of eight groups 8.8, but tiles that fill the CUs twice take 1.7 times as long
// then; 16 tiles of 64 x 64 22 us, with two groups 15, with four 14).
template <typename D, int TILE> struct LossTiles;
template <typename D> struct LossTiles<D, 256> { static constexpr int M = 256, N = 256, WM = 2, WN = 4, kGroups = 1; };
template <typename D> struct LossTiles<D, 128> { static constexpr int M = 128, N = 128, WM = 2, WN = 2, kGroups = 1; };
template <typename D> struct LossTiles<D, 64> { static constexpr int M = 64, N = 64, WM = 2, WN = 2, kGroups = 1; };
template <typename D> struct LossTiles<D, 32> { static constexpr int M = 32, N = 32, WM = 1, WN = 1, kGroups = 4; };
template <typename D, int TILE, bool A_ACROSS, bool B_ACROSS>
using LossProduct = Product<D, LossTiles<D, TILE>::M, LossTiles<D, TILE>::N, LossTiles<D, TILE>::WM, LossTiles<D, TILE>::WN, A_ACROSS, B_ACROSS, LossTiles<D, TILE>::kGroups>;

// z[v][row] = W[v] . H[row].  Bound by the matrix cores' power and, where the width is small, by what comes behind the products: an exponential is a quarter of the vector unit's rate, and a tile's end takes
// as long as seven stages of 64 (4096 rows, 4096 wide, 32000 words in bf16 0.81 ms, 1330 TFLOP/s; 1800 x 1000 x 50021 in fp16 0.28 ms, 650).
template <typename D, int TILE>
__global__ __launch_bounds__((LossProduct<D, TILE, false, false>::kThreads)) void k_loss_logits(LossArgs a) {
    using P = LossProduct<D, TILE, false, false>;
    extern __shared__ uint8_t lds_bytes[];
    const Lds lds = (Lds)lds_bytes;
    const int rows = rows_of_block(a);
    const uint32_t tiles_m = a.padded / P::BM, tiles_n = (rows + P::BN - 1) / P::BN, item = item_of_block(blockIdx.x, tiles_m * tiles_n);
    if (item == tiles_m * tiles_n) return;
    uint32_t tm, tn;
    tile_of_item(item, tiles_m, tiles_n, tm, tn);
    const int v0 = tm * P::BM, r0 = tn * P::BN;
    const int64_t w_bytes = a.w_stride * D::size, h_bytes = (int64_t)a.width * D::size;
    P p;
    if (!p.run({static_cast<const uint8_t*>(a.W) + v0 * w_bytes, w_bytes}, {a.packed + r0 * h_bytes, h_bytes}, a.width, max(a.vocab - v0, 0), P::BN, lds)) return;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, wm = wave % P::WM, wn = wave / P::WM, g = lane >> 4;
    const int first = v0 + wm * P::kRange;                                                // of the wave's piece
    const int64_t piece = first / P::kRange;
#pragma unroll
    for (int j = 0; j < P::NI; ++j) {
        const int row = r0 + 16 * (wn * P::NI + j) + (lane & 15);
        const int want = a.target[row] - first - 4 * g;                                   // (a lane has v = first + 4 g + 16 i + 0..3)
        float plain = 0.0f;
        if (__any(want >= 0 && want < P::kRange)) {                                       // (few pieces have the target of any of 16 rows)
            float hit = 0.0f;
#pragma unroll
            for (int i = 0; i < P::MI; ++i)
#pragma unroll
                for (int x = 0; x < 4; ++x) hit = want == 16 * i + x ? p.acc[j][i][x] : hit;
            if (want >= 0 && want < P::kRange && (want & 12) == 0) a.hit[row] = hit;
        }
        if (a.smoothing > 0.0f) {                                                         // (z behind the vocabulary is 0)
#pragma unroll
            for (int i = 0; i < P::MI; ++i)
#pragma unroll
                for (int x = 0; x < 4; ++x) plain += p.acc[j][i][x];
            plain = quarters_sum(plain);
            if (g == 0) a.plain[piece * a.block_rows + row] = plain;
        }
        if (first + P::kRange > a.vocab) {
#pragma unroll
            for (int i = 0; i < P::MI; ++i)
#pragma unroll
                for (int x = 0; x < 4; ++x) p.acc[j][i][x] = first + 4 * g + 16 * i + x < a.vocab ? p.acc[j][i][x] : -INFINITY;
        }
        float top = -INFINITY, sum = 0.0f;
#pragma unroll
        for (int i = 0; i < P::MI; ++i)
#pragma unroll
            for (int x = 0; x < 4; ++x) top = fmaxf(top, p.acc[j][i][x]);
        top = quarters_max(top);
        // (The maximum is taken off first: near it that has no rounding, however large both are.)
        const float base = top == -INFINITY ? 0.0f : top;
#pragma unroll
        for (int i = 0; i < P::MI; ++i)
#pragma unroll
            for (int x = 0; x < 4; ++x) p.acc[j][i][x] = __builtin_amdgcn_exp2f(fmaf(p.acc[j][i][x] - base, kLossLog2e, kLossTopLog2<D>));
#pragma unroll
        for (int i = 0; i < P::MI; ++i)
#pragma unroll
            for (int x = 0; x < 4; ++x) sum += p.acc[j][i][x];
        sum = quarters_sum(sum) * (1.0f / kLossTop<D>);
        if (g == 0) { a.top[piece * a.block_rows + row] = top; a.sum[piece * a.block_rows + row] = sum; }
    }
    if (!a.train) return;
#pragma unroll
    for (int j = 0; j < P::NI; j += 2) {
        const int row0 = r0 + 16 * (wn * P::NI + j);
        store_two_blocks<LossExp<D>, P::MI>(p.acc + j, 1.0f, lds + wave * (32 * P::kRange * D::size), P::kRange, lane,
                                   [&](uint32_t r) { return a.e + ((int64_t)(row0 + (int)r) * a.padded + first) * D::size; });
    }
}

// dH[row][d] = sum over v of dz[row][v] W[v][d]; with several parts of the vocabulary each has its sum in fp32
template <typename D, int TILE> __device__ __forceinline__ void loss_dh(const LossArgs& a, uint32_t block, Lds lds) {
    using P = LossProduct<D, TILE, true, false>;
    const int rows = rows_of_block(a);
    const LossParts parts = parts_of_dh(a, rows);
    const uint32_t tiles_m = (a.width + P::BM - 1) / P::BM, tiles_n = (rows + P::BN - 1) / P::BN, items = tiles_m * tiles_n * parts.splits, item = item_of_block(block, items);
    if (item == items) return;
    const uint32_t split = item / (tiles_m * tiles_n);
    uint32_t tm, tn;
    tile_of_item(item - split * tiles_m * tiles_n, tiles_m, tiles_n, tm, tn);
    const int d0 = tm * P::BM, r0 = tn * P::BN, steps = (a.vocab + P::BK - 1) / P::BK, share = (steps + parts.splits - 1) / parts.splits;
    const int v0 = min((int)split * share * P::BK, a.vocab), v1 = min(v0 + share * P::BK, a.vocab);
    const int64_t w_bytes = a.w_stride * D::size, e_bytes = (int64_t)a.padded * D::size;
    P p;
    if (!p.run({static_cast<const uint8_t*>(a.W) + v0 * w_bytes + (int64_t)d0 * D::size, w_bytes}, {a.e + r0 * e_bytes + (int64_t)v0 * D::size, e_bytes}, v1 - v0, a.width - d0, P::BN, lds)) return;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, wm = wave % P::WM, wn = wave / P::WM;
    const int first = d0 + wm * P::kRange, left = a.width - first;
    const float factor = 1.0f / gradient_scale<D>(a);
    if constexpr (D::size == 2) {
        // what the rounding of a target's dz took off, times its row of W; with several parts k_loss_dh_sum adds it
        if (a.dh_splits == 1) {
#pragma unroll
            for (int j = 0; j < P::NI; ++j) {
                const int row = min(r0 + 16 * (wn * P::NI + j) + (lane & 15), rows - 1), d = first + 4 * (lane >> 4);
                const float x = a.left[row];
                const uint8_t* const w = static_cast<const uint8_t*>(a.W) + a.target[row] * w_bytes;
#pragma unroll
                for (int i = 0; i < P::MI; ++i) p.acc[j][i] += x * four_of<D>(w + min(d + 16 * i, a.width - 4) * D::size);
            }
        }
    }
#pragma unroll
    for (int j = 0; j < P::NI; j += 2) {
        const int row0 = r0 + 16 * (wn * P::NI + j);
        if (a.dh_splits > 1) {
            float* const to = a.dh_parts + (int64_t)split * parts.rows * a.width + first;
            store_two_blocks<F32, P::MI>(p.acc + j, factor, lds + wave * (32 * P::kRange * 4), left, lane,
                                         [&](uint32_t r) { return reinterpret_cast<uint8_t*>(to + (int64_t)(row0 + (int)r) * a.width); });
        } else {
            store_two_blocks<D, P::MI>(p.acc + j, factor, lds + wave * (32 * P::kRange * D::size), left, lane, [&](uint32_t r) -> uint8_t* {
                const int row = row0 + (int)r;
                return row < rows ? static_cast<uint8_t*>(a.dH) + (a.index[a.block * a.block_rows + row] * a.dh_stride + first) * D::size : nullptr;
            });
        }
    }
}

// dW[v][d] = sum over the rows of dz[row][v] H[row][d]
template <typename D, int TILE> __device__ __forceinline__ void loss_dw(const LossArgs& a, uint32_t block, Lds lds) {
    using P = LossProduct<D, TILE, true, true>;
    const int rows = rows_of_block(a);
    const uint32_t tiles_m = (a.width + P::BM - 1) / P::BM, tiles_n = (a.vocab + P::BN - 1) / P::BN, item = item_of_block(block, tiles_m * tiles_n);
    if (item == tiles_m * tiles_n) return;
    uint32_t tm, tn;
    tile_of_item(item, tiles_m, tiles_n, tm, tn);
    const int d0 = tm * P::BM, v0 = tn * P::BN;
    const int64_t h_bytes = (int64_t)a.width * D::size, e_bytes = (int64_t)a.padded * D::size;
    P p;
    // (up to whole steps: the rows behind those that count are zeros in both)
    if (!p.run({a.packed + (int64_t)d0 * D::size, h_bytes}, {a.e + (int64_t)v0 * D::size, e_bytes}, (rows_of_dw(a, rows) + P::BK - 1) / P::BK * P::BK, a.width - d0, P::BN, lds)) return;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, wm = wave % P::WM, wn = wave / P::WM;
    const int first = d0 + wm * P::kRange, left = a.width - first;
    const float factor = 1.0f / gradient_scale<D>(a);
#pragma unroll
    for (int j = 0; j < P::NI; j += 2) {
        const int row0 = v0 + 16 * (wn * P::NI + j);
        if (a.blocks > 1) {
            // the sum so far is added in registers: a lane has four d that follow one another
            float* const so_far = D::size == 4 ? static_cast<float*>(a.dW) : a.dw_sum;
            const int64_t stride = D::size == 4 ? a.dw_stride : a.width;
#pragma unroll
            for (int jj = j; jj < j + 2; ++jj)
#pragma unroll
                for (int i = 0; i < P::MI; ++i) {
                    const int v = row0 + 16 * (jj - j) + (lane & 15), d = first + 16 * i + 4 * (lane >> 4);
                    f32x4 x = p.acc[jj][i] * factor;
                    if (v < a.vocab && d < a.width) {
                        f32x4* const at = reinterpret_cast<f32x4*>(so_far + v * stride + d);
                        if (a.block > 0) x += *at;
                        if (D::size == 4 || a.block + 1 < a.blocks) *at = x;
                        else store_four<D>(static_cast<uint8_t*>(a.dW) + (v * a.dw_stride + d) * D::size, x[0], x[1], x[2], x[3]);
                    }
                }
        } else {
            store_two_blocks<D, P::MI>(p.acc + j, factor, lds + wave * (32 * P::kRange * D::size), left, lane, [&](uint32_t r) -> uint8_t* {
                const int v = row0 + (int)r;
                return v < a.vocab ? static_cast<uint8_t*>(a.dW) + (v * a.dw_stride + first) * D::size : nullptr;
            });
        }
    }
}

// Both gradients in one launch: the longer products first (as a rule dH's, over the vocabulary), and the others where those leave room.  All of a call, each gradient with its own launch and its
// own tile, and so: 1000 rows, width 1024, 8000 words in bf16 105 and 86 us, 128 x 1024 x 128000 286 and 246, 64 x 256 x 1000 in fp32 35.9 and 32.1; 6000 x 640 x 3000, where dW's products are the longer ones,
// 158 and 151 (dH's first: 183).
template <typename D, int TILE>
__global__ __launch_bounds__((LossProduct<D, TILE, true, true>::kThreads)) void k_loss_back(LossArgs a) {
    extern __shared__ uint8_t lds_bytes[];
    const bool first = (int)blockIdx.x < a.first_blocks;
    const uint32_t block = first ? blockIdx.x : blockIdx.x - a.first_blocks;
    if (first != (a.dw_first != 0)) loss_dh<D, TILE>(a, block, (Lds)lds_bytes);
    else loss_dw<D, TILE>(a, block, (Lds)lds_bytes);
}

template <typename P, auto Kernel> static inline hipError_t launch_tiles(const LossArgs& a, uint32_t tiles, hipStream_t st) {
    const hipError_t e = allow_dynamic_lds<Kernel, P::kLds>();
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(Kernel, dim3(tiles), dim3(P::kThreads), P::kLds, st, a);
    return hipGetLastError();
}
template <typename D, int TILE> static inline hipError_t launch_logits_of(const LossArgs& a, hipStream_t st) {
    return launch_tiles<LossProduct<D, TILE, false, false>, &k_loss_logits<D, TILE>>(a, (uint32_t)(a.padded / TILE * (a.block_rows / TILE)), st);
}
template <typename D, int TILE> static inline hipError_t launch_back_of(LossArgs a, hipStream_t st) {
    const int tiles = (a.width + TILE - 1) / TILE;
    const int dh = a.dH ? (tiles * a.dh_room + 7) / 8 * 8 : 0, dw = a.dW ? (tiles * ((a.vocab + TILE - 1) / TILE) + 7) / 8 * 8 : 0;   // (of eight, so that both begin at the first XCD)
    a.first_blocks = a.dw_first ? dw : dh;
    return launch_tiles<LossProduct<D, TILE, true, true>, &k_loss_back<D, TILE>>(a, (uint32_t)(dh + dw), st);
}
// (fp32: fragments of 256 x 256 tiles would not find room in the registers)
template <typename D, typename Launch> static inline hipError_t with_tile(int tile, Launch&& launch) {
    using std::integral_constant;
    if constexpr (D::size == 2) if (tile == 256) return launch(integral_constant<int, 256>{});
    return tile == 128 ? launch(integral_constant<int, 128>{}) : tile == 64 ? launch(integral_constant<int, 64>{}) : launch(integral_constant<int, 32>{});
}
template <typename D> hipError_t launch_loss_logits(const LossArgs& a, hipStream_t st) {
    return with_tile<D>(a.tile[0], [&](auto tile) { return launch_logits_of<D, tile()>(a, st); });
}
template <typename D> hipError_t launch_loss_back(const LossArgs& a, hipStream_t st) {
    return with_tile<D>(a.tile[1], [&](auto tile) { return launch_back_of<D, tile()>(a, st); });
}
#endif

}  // namespace lsp

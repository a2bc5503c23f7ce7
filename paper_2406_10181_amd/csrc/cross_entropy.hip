// Cross entropy: which rows count, the rows' losses, the gradient of z, and the plan.  The products are in cross_entropy.h.
#include <algorithm>
#include <cmath>

#include "cross_entropy.h"
#include "rows.h"

namespace lsp {

constexpr int kIndexThreads = 1024, kIndexRows = 4;                      // rows of a thread at a time

// The rows that count, in order, and how many; one workgroup (the rows' targets are a few bytes each)
__global__ __launch_bounds__(kIndexThreads) void k_loss_index(LossArgs a) {
    __shared__ int waves[kIndexThreads / 64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int found = 0;
    for (int64_t base = 0; base < a.rows; base += kIndexThreads * kIndexRows) {
        bool counts[kIndexRows];
        int mine = 0;
#pragma unroll
        for (int k = 0; k < kIndexRows; ++k) {
            const int64_t row = base + threadIdx.x * kIndexRows + k;
            const int64_t target = row < a.rows ? a.targets[row] : -1;
            counts[k] = target >= 0 && target < a.vocab;
            mine += counts[k];
        }
        int before = mine;                                               // of this lane and those below
#pragma unroll
        for (int d = 1; d < 64; d *= 2) {
            const int x = __shfl_up(before, d);
            if (lane >= d) before += x;
        }
        if (lane == 63) waves[wave] = before;
        __syncthreads();
        int at = found + before - mine;
#pragma unroll
        for (int w = 0; w < kIndexThreads / 64; ++w) {
            if (w < wave) at += waves[w];
            found += waves[w];
        }
#pragma unroll
        for (int k = 0; k < kIndexRows; ++k)
            if (counts[k]) a.index[at++] = (int)(base + threadIdx.x * kIndexRows + k);
        __syncthreads();
    }
    if (threadIdx.x == 0) { a.count[0] = found; a.count[1] = 0; }
}

// Workgroups below block_rows: a row of the block's packed rows, zeros behind the last one up to a whole tile.  Workgroups from there on (first block only): a row
// that does not count gets its zeros.
__global__ __launch_bounds__(256) void k_loss_pack(LossArgs a, int row_bytes, int elem) {
    const int rows = rows_of_block(a);
    if ((int)blockIdx.x < a.block_rows) {
        const int slot = blockIdx.x;
        if (slot >= (rows + 255) / 256 * 256) return;
        u32x4* const to = reinterpret_cast<u32x4*>(a.packed + (int64_t)slot * row_bytes);
        if (slot < rows) {
            const int64_t row = a.index[a.block * a.block_rows + slot];
            const u32x4* const from = reinterpret_cast<const u32x4*>(static_cast<const uint8_t*>(a.H) + row * a.h_stride * elem);
            for (int k = threadIdx.x; k < row_bytes / 16; k += 256) to[k] = from[k];
            if (threadIdx.x == 0) a.target[slot] = (int)a.targets[row];
        } else {
            for (int k = threadIdx.x; k < row_bytes / 16; k += 256) to[k] = u32x4{0, 0, 0, 0};
            if (threadIdx.x == 0) a.target[slot] = -1;
        }
        return;
    }
    const int64_t row = blockIdx.x - a.block_rows;
    const int64_t target = a.targets[row];
    if (target >= 0 && target < a.vocab) return;
    if (threadIdx.x == 0) {
        a.losses[row] = 0.0f;
        if (a.logs) a.logs[row] = 0.0f;
    }
    if (!a.dH) return;
    u32x4* const to = reinterpret_cast<u32x4*>(static_cast<uint8_t*>(a.dH) + row * a.dh_stride * elem);
    for (int k = threadIdx.x; k < row_bytes / 16; k += 256) to[k] = u32x4{0, 0, 0, 0};
}

// Both of these for few rows, in one launch: a workgroup has a row (or, from `rows` on, a row of zeros behind the packed ones) and counts those before it itself.
constexpr int kFewRows = 2048;
__global__ __launch_bounds__(256) void k_loss_pack_few(LossArgs a, int row_bytes, int elem) {
    __shared__ int waves[4][2];
    const int row = (int)min((int64_t)blockIdx.x, a.rows), rows = (int)a.rows;
    int before = 0, all = 0;
    for (int k = threadIdx.x; k < rows; k += 256) {
        const int64_t t = a.targets[k];
        const bool counts = t >= 0 && t < a.vocab;
        before += counts && k < row;
        all += counts;
    }
#pragma unroll
    for (int d = 32; d; d /= 2) { before += __shfl_xor(before, d); all += __shfl_xor(all, d); }
    if ((threadIdx.x & 63) == 0) { waves[threadIdx.x >> 6][0] = before; waves[threadIdx.x >> 6][1] = all; }
    __syncthreads();
    before = waves[0][0] + waves[1][0] + waves[2][0] + waves[3][0];
    all = waves[0][1] + waves[1][1] + waves[2][1] + waves[3][1];
    if (blockIdx.x == 0 && threadIdx.x == 0) { a.count[0] = all; a.count[1] = 0; }
    const u32x4* from = nullptr;
    u32x4* to = nullptr;
    if ((int)blockIdx.x < rows) {
        const int64_t target = a.targets[row];
        if (target >= 0 && target < a.vocab) {
            from = reinterpret_cast<const u32x4*>(static_cast<const uint8_t*>(a.H) + row * a.h_stride * elem);
            to = reinterpret_cast<u32x4*>(a.packed + (int64_t)before * row_bytes);
            if (threadIdx.x == 0) { a.index[before] = row; a.target[before] = (int)target; }
        } else {
            if (threadIdx.x == 0) {
                a.losses[row] = 0.0f;
                if (a.logs) a.logs[row] = 0.0f;
            }
            if (a.dH) to = reinterpret_cast<u32x4*>(static_cast<uint8_t*>(a.dH) + row * a.dh_stride * elem);
        }
    } else {
        const int slot = all + (int)blockIdx.x - rows;
        if (slot >= (all + 255) / 256 * 256) return;
        to = reinterpret_cast<u32x4*>(a.packed + (int64_t)slot * row_bytes);
        if (threadIdx.x == 0) a.target[slot] = -1;
    }
    if (!to) return;
    for (int k = threadIdx.x; k < row_bytes / 16; k += 256) to[k] = from ? from[k] : u32x4{0, 0, 0, 0};
}

// L and the loss of a row from its pieces: 16 rows a workgroup, RUNS threads a row, each a running maximum and sum
template <int RUNS>
__global__ __launch_bounds__(16 * RUNS) void k_loss_rows(LossArgs a, int fp16) {
    __shared__ float tops[RUNS][17], sums[RUNS][17], plains[RUNS][17];
    const int rows = rows_of_block(a), run = threadIdx.x >> 4, r = threadIdx.x & 15, row = blockIdx.x * 16 + r;
    if ((int)blockIdx.x * 16 >= rows) return;
    float top = -INFINITY, sum = 0.0f, plain = 0.0f;
    // (rows behind the last: the pieces are there, of packed zeros or of nothing yet, and nothing is made of them)
    if (row < rows) {
#pragma unroll 4
        for (int p = run; p < a.pieces; p += RUNS) {
            const int64_t at = (int64_t)p * a.block_rows + row;
            const float t = a.top[at], s = a.sum[at], higher = fmaxf(top, t), from = higher == -INFINITY ? 0.0f : higher;
            sum = sum * __builtin_amdgcn_exp2f((top - from) * kLossLog2e) + s * __builtin_amdgcn_exp2f((t - from) * kLossLog2e);
            top = higher;
            if (a.smoothing > 0.0f) plain += a.plain[at];
        }
    }
    tops[run][r] = top; sums[run][r] = sum; plains[run][r] = plain;
    __syncthreads();
    float bound = 0.0f;
    if (run == 0 && row < rows) {
#pragma unroll 16
        for (int k = 1; k < RUNS; ++k) top = fmaxf(top, tops[k][r]);
        const float from = top == -INFINITY ? 0.0f : top;
        sum = plain = 0.0f;
#pragma unroll 16
        for (int k = 0; k < RUNS; ++k) {
            sum += sums[k][r] * __builtin_amdgcn_exp2f((tops[k][r] - from) * kLossLog2e);
            plain += plains[k][r];
        }
        const float L = top + logf(sum);
        float loss = L - (1.0f - a.smoothing) * a.hit[row];
        if (a.smoothing > 0.0f) loss -= a.smoothing * (plain / (float)a.vocab);
        if (a.z_loss > 0.0f) loss = fmaf(a.z_loss * L, L, loss);
        const int64_t to = a.index[a.block * a.block_rows + row];
        a.losses[to] = loss;
        if (a.logs) a.logs[to] = L;
        if (a.train) {
            const float factor = a.weights ? a.scale * a.weights[to] : a.scale;
            a.log_sum[row] = L;
            a.factor[row] = factor;
            bound = fabsf(factor) * fmaf(2.0f * a.z_loss, fabsf(L), 2.0f);
        }
    }
    if (!fp16 || !a.train || run) return;
    // the largest gradient of z that there can be: 16 lanes' maximum, and an atomic one, whose order is of no matter.  (What is not finite has no say.)
    bound = bound <= 3.402823466e38f ? bound : 0.0f;
#pragma unroll
    for (int d = 8; d; d /= 2) bound = fmaxf(bound, __shfl_xor(bound, d));
    if (r == 0) atomicMax(reinterpret_cast<unsigned*>(a.count) + 1, __float_as_uint(bound));
}

constexpr int kDzColumns = 512;                                          // of a workgroup of k_loss_dz, in steps of 128

// dz = (p (1 + 2 z_loss L) - smoothing / vocab - (1 - smoothing) [v = target]) factor in place of the exponentials: 16 rows a workgroup, so that the pieces' maxima come in
// whole lines.  Two bytes read and two written an element: bound by memory.
template <typename D>
__global__ __launch_bounds__(256) void k_loss_dz(LossArgs a) {
    const int rows = rows_of_block(a), chunks = (a.padded + kDzColumns - 1) / kDzColumns;
    const int row = (int)(blockIdx.x / chunks) * 16 + (threadIdx.x >> 4), v0 = (int)(blockIdx.x % chunks) * kDzColumns + (threadIdx.x & 15) * 8;
    if (row >= (rows + 63) / 64 * 64) return;
    typename D::elem* const e = reinterpret_cast<typename D::elem*>(a.e) + (int64_t)row * a.padded;
    const bool there = row < rows;
    const float L = there ? a.log_sum[row] : 0.0f, factor = there ? a.factor[row] * gradient_scale<D>(a) : 0.0f;
    const float share = a.smoothing / (float)a.vocab, rise = fmaf(2.0f * a.z_loss, L, 1.0f);
    const int target = there ? a.target[row] : -1;
#pragma unroll 4
    for (int c = 0; c < kDzColumns; c += 128) {
        const int v = v0 + c;
        if (v >= a.padded) break;
        Eight x;
        if (there) {
            x = load_eight<D>(e + v, 8);
            const float of_piece = a.top[(int64_t)(v / a.piece) * a.block_rows + row];
            const float by = __builtin_amdgcn_exp2f((of_piece - L) * kLossLog2e) * (1.0f / kLossTop<D>) * rise * factor;
#pragma unroll
            for (int k = 0; k < 8; ++k) x.x[k] = v + k < a.vocab ? fmaf(x.x[k], by, -share * factor) : 0.0f;
            if (target >= v && target < v + 8) {
                // of the target z is there in fp32: p - 1 without what the rounding of p would leave of it
                const float p_less_1 = expm1f(a.hit[row] - L), there_now = (p_less_1 * rise + (rise - 1.0f) + a.smoothing - share) * factor;
#pragma unroll
                for (int k = 0; k < 8; ++k) x.x[k] = v + k == target ? there_now : x.x[k];
            }
        } else {
#pragma unroll
            for (int k = 0; k < 8; ++k) x.x[k] = 0.0f;
        }
        store_eight<D>(e + v, x, 8);
    }
}

// The parts of dH, added in their order
template <typename D>
__global__ __launch_bounds__(256) void k_loss_dh_sum(LossArgs a) {
    const int rows = rows_of_block(a), units = a.width / 4;
    const int64_t n = (int64_t)blockIdx.x * 256 + threadIdx.x;
    const int row = (int)(n / units), d = (int)(n - (int64_t)row * units) * 4;
    if (row >= rows) return;
    const LossParts parts = parts_of_dh(a, rows);
    f32x4 sum = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll 8
    for (int s = 0; s < parts.splits; ++s) sum += *reinterpret_cast<const f32x4*>(a.dh_parts + ((int64_t)s * parts.rows + row) * a.width + d);
    store_four<D>(static_cast<uint8_t*>(a.dH) + (a.index[a.block * a.block_rows + row] * a.dh_stride + d) * D::size, sum[0], sum[1], sum[2], sum[3]);
}

// ------------------------------------------------------------------ plan
static int64_t ceil_to(int64_t x, int64_t to) { return (x + to - 1) / to * to; }

// The time of tiles of m x n products over `length`, in us, by a rough account: operations a us of a CU whose workgroups are few in all (fewer than half the CUs: clocks are higher then), of
// one among many, and of as many as it holds; and what a round of them costs besides.  Measured in bf16 with tiles of 256, 128 and 64, logits: rows 1000, width 512, vocabulary 4000: 19, 12.5
// and 12 us; 1000, 1024, 8000: 30, 25.5 and 32; 1000, 1024, 32000: 68, 92 and 121; 64, 1024, 32000: 31, 19 and 14.
struct TileRate { int tile, at_once; double few, one, all, round; };
constexpr TileRate kTileRates[3] = {{256, 1, 7.5e6, 4.8e6, 4.8e6, 5.0}, {128, 2, 3.3e6, 2.6e6, 3.6e6, 3.0}, {64, 4, 1.35e6, 1.0e6, 2.6e6, 2.0}};
constexpr TileRate kTileRatesF32[2] = {{128, 2, 0.49e6, 0.49e6, 0.5e6, 3.0}, {64, 4, 0.39e6, 0.39e6, 0.52e6, 2.0}};   // (256: its fragments would not find room in the registers)
static double products_us(int64_t m, int64_t n, int64_t length, const TileRate& r, int splits) {
    const int64_t tiles = (m + r.tile - 1) / r.tile * ((n + r.tile - 1) / r.tile) * splits;
    const int here = (int)std::min<int64_t>(r.at_once, (tiles + 255) / 256);
    const double rate = tiles <= 128 ? r.few : std::min(here * r.one, r.all);
    return (double)((tiles + 256 * here - 1) / (256 * here)) * (r.round + here * 2.0 * r.tile * r.tile * (double)((length + splits - 1) / splits) / rate);
}
// The tile and the number of parts of `length` (at most `most`) that take the least; parts' sums are written and read again, at 5 TB/s, by a launch more
static void best_tile(int64_t m, int64_t n, int64_t length, bool fp32, int most, int32_t& tile, int32_t& splits) {
    double least = 1e30;
    const TileRate* const rates = fp32 ? kTileRatesF32 : kTileRates;
    for (int k = 0; k < (fp32 ? 2 : 3); ++k)
        for (int s = 1; s <= most; ++s) {
            const double us = products_us(m, n, length, rates[k], s) + (s > 1 ? 4.0 + 1.6e-6 * (double)s * (double)(m * n) : 0.0);
            if (us < least) { least = us; tile = rates[k].tile; splits = s; }
        }
}

void plan_loss(LossArgs& a, lsp_dtype dtype) {
    const bool fp32 = dtype == LSP_F32;
    const int64_t size = fp32 ? 4 : 2;
    a.padded = (int)ceil_to(a.vocab, 256);
    const int64_t row = std::max<int64_t>(a.width, a.train ? a.padded : 0) * size;
    const int64_t most = std::max<int64_t>(256, std::min<int64_t>((int64_t)kLossBytes / row, a.train ? LSP_MAX_ROWS : 16384) / 256 * 256);
    a.blocks = (int)((a.rows + most - 1) / most);
    a.block_rows = (int)ceil_to((a.rows + a.blocks - 1) / a.blocks, 256);
    a.blocks = (int)((a.rows + a.block_rows - 1) / a.block_rows);
    const int64_t rows = std::min<int64_t>(a.rows, a.block_rows);
    int32_t whole;
    best_tile(a.vocab, rows, a.width, fp32, 1, a.tile[0], whole);
    a.piece = a.tile[0] / 2;
    a.pieces = a.padded / a.piece;
    best_tile(a.width, rows, a.vocab, fp32, 32, a.tile[1], a.dh_splits);
    a.dh_room = (int)((rows + a.tile[1] - 1) / a.tile[1]) * a.dh_splits;
    best_tile(a.width, a.vocab, rows, fp32, 1, a.tile[2], whole);
}

size_t loss_workspace(LossArgs& a, lsp_dtype dtype, uint8_t* base) {
    const size_t size = dtype == LSP_F32 ? 4 : 2;
    size_t total = 0;
    const auto take = [&](auto& p, size_t bytes) {
        using T = std::remove_reference_t<decltype(p)>;
        if (base) p = reinterpret_cast<T>(base + total);
        total += align_up(bytes, 256);
    };
    take(a.count, 16);
    take(a.index, (size_t)a.rows * 4);
    take(a.packed, (size_t)a.block_rows * a.width * size);
    take(a.target, (size_t)a.block_rows * 4);
    take(a.top, (size_t)a.pieces * a.block_rows * 4);
    take(a.sum, (size_t)a.pieces * a.block_rows * 4);
    take(a.plain, a.smoothing > 0.0f ? (size_t)a.pieces * a.block_rows * 4 : 0);
    take(a.hit, (size_t)a.block_rows * 4);
    if (a.train) {
        take(a.log_sum, (size_t)a.block_rows * 4);
        take(a.factor, (size_t)a.block_rows * 4);
        take(a.e, (size_t)a.block_rows * a.padded * size);
        take(a.dh_parts, a.dh_splits > 1 ? (size_t)a.dh_splits * a.block_rows * a.width * 4 : 0);
        take(a.dw_sum, a.blocks > 1 && size == 2 ? (size_t)a.vocab * a.width * 4 : 0);
    }
    return total;
}

template <typename D> static hipError_t launch_blocks(LossArgs& a, lsp_dtype dtype, hipStream_t st) {
    const bool few = a.rows <= kFewRows && a.blocks == 1;
    const int row_bytes = a.width * D::size;
    if (few) hipLaunchKernelGGL(k_loss_pack_few, dim3((unsigned)(a.rows + 255)), dim3(256), 0, st, a, row_bytes, (int)D::size);
    else hipLaunchKernelGGL(k_loss_index, dim3(1), dim3(kIndexThreads), 0, st, a);
    hipError_t e = hipGetLastError();
    for (a.block = 0; a.block < a.blocks && e == hipSuccess; ++a.block) {
        if (!few) hipLaunchKernelGGL(k_loss_pack, dim3((unsigned)(a.block_rows + (a.block == 0 ? a.rows : 0))), dim3(256), 0, st, a, row_bytes, (int)D::size);
        if ((e = hipGetLastError()) != hipSuccess || (e = launch_loss_logits<D>(a, st)) != hipSuccess) break;
        if (a.pieces > 64) hipLaunchKernelGGL(k_loss_rows<64>, dim3((unsigned)(a.block_rows / 16)), dim3(1024), 0, st, a, (int)std::is_same<D, F16>::value);
        else hipLaunchKernelGGL(k_loss_rows<16>, dim3((unsigned)(a.block_rows / 16)), dim3(256), 0, st, a, (int)std::is_same<D, F16>::value);
        if ((e = hipGetLastError()) != hipSuccess || !a.train) continue;
        hipLaunchKernelGGL(k_loss_dz<D>, dim3((unsigned)(a.block_rows / 16 * ((a.padded + kDzColumns - 1) / kDzColumns))), dim3(256), 0, st, a);
        if ((e = hipGetLastError()) != hipSuccess) break;
        if (a.dH) {
            if ((e = launch_loss_dh<D>(a, st)) != hipSuccess) break;
            if (a.dh_splits > 1) {
                hipLaunchKernelGGL(k_loss_dh_sum<D>, dim3((unsigned)(((int64_t)a.block_rows * (a.width / 4) + 255) / 256)), dim3(256), 0, st, a);
                if ((e = hipGetLastError()) != hipSuccess) break;
            }
        }
        if (a.dW) e = launch_loss_dw<D>(a, st);
    }
    return e;
}

hipError_t launch_loss(LossArgs& a, lsp_dtype dtype, hipStream_t st) {
    return dtype == LSP_F32 ? launch_blocks<F32>(a, dtype, st) : dtype == LSP_F16 ? launch_blocks<F16>(a, dtype, st) : launch_blocks<BF16>(a, dtype, st);
}

}  // namespace lsp

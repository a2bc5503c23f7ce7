// Cross entropy: which rows count, the rows' losses, the gradient of z, and the plan.  The products are in cross_entropy_products.h.
#include <algorithm>
#include <cmath>

#include "cross_entropy.h"
#include "rows.h"

namespace lsp {

// The largest of 64 lanes' numbers, in all of them
__device__ __forceinline__ float top_of_wave(float x) {
#pragma unroll
    for (int d = 32; d; d /= 2) x = fmaxf(x, __shfl_xor(x, d));
    return x;
}
// A row's part in the largest weight (of what is not finite none)
__device__ __forceinline__ float weight_of(const LossArgs& a, int64_t row) {
    const float w = a.weights ? fabsf(a.weights[row]) : 1.0f;
    return w <= 3.402823466e38f ? w : 0.0f;
}

constexpr int kIndexThreads = 1024, kIndexRows = 4;                      // rows of a thread at a time

// The rows that count, in order, and how many; one workgroup (the rows' targets are a few bytes each)
__global__ __launch_bounds__(kIndexThreads) void k_loss_index(LossArgs a) {
    __shared__ int waves[kIndexThreads / 64];
    __shared__ float tops[kIndexThreads / 64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int found = 0;
    float top = 0.0f;
    for (int64_t base = 0; base < a.rows; base += kIndexThreads * kIndexRows) {
        bool counts[kIndexRows];
        int mine = 0;
#pragma unroll
        for (int k = 0; k < kIndexRows; ++k) {
            const int64_t row = base + threadIdx.x * kIndexRows + k;
            const int64_t target = row < a.rows ? a.targets[row] : -1;
            counts[k] = target >= 0 && target < a.vocab;
            mine += counts[k];
            if (counts[k]) top = fmaxf(top, weight_of(a, row));
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
    top = top_of_wave(top);
    if (lane == 0) tops[wave] = top;
    __syncthreads();
    if (wave) return;
    top = top_of_wave(lane < kIndexThreads / 64 ? tops[lane] : 0.0f);
    if (lane == 0) { a.count[0] = found; a.count[1] = 0; a.count[2] = __float_as_int(top); }
}

// (4096 rows of 4096 in bf16: 15.6 us, 4.3 TB/s.)  Workgroups below block_rows: a row of the block's packed rows, zeros behind the last one up to a whole tile.  Workgroups from there on (first block only): a row
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
    __shared__ float tops[4];
    const int row = (int)min((int64_t)blockIdx.x, a.rows), rows = (int)a.rows;
    int before = 0, all = 0;
    float top = 0.0f;
    for (int k = threadIdx.x; k < rows; k += 256) {
        const int64_t t = a.targets[k];
        const bool counts = t >= 0 && t < a.vocab;
        before += counts && k < row;
        all += counts;
        if (blockIdx.x == 0 && counts) top = fmaxf(top, weight_of(a, k));
    }
    if (blockIdx.x == 0) {
        top = top_of_wave(top);
        if ((threadIdx.x & 63) == 0) tops[threadIdx.x >> 6] = top;
    }
#pragma unroll
    for (int d = 32; d; d /= 2) { before += __shfl_xor(before, d); all += __shfl_xor(all, d); }
    if ((threadIdx.x & 63) == 0) { waves[threadIdx.x >> 6][0] = before; waves[threadIdx.x >> 6][1] = all; }
    __syncthreads();
    before = waves[0][0] + waves[1][0] + waves[2][0] + waves[3][0];
    all = waves[0][1] + waves[1][1] + waves[2][1] + waves[3][1];
    if (blockIdx.x == 0 && threadIdx.x == 0) { a.count[0] = all; a.count[1] = 0; a.count[2] = __float_as_int(fmaxf(fmaxf(tops[0], tops[1]), fmaxf(tops[2], tops[3]))); }
    const u32x4* from = nullptr;
    u32x4 *to = nullptr, *again = nullptr;
    if ((int)blockIdx.x < rows) {
        const int64_t target = a.targets[row];
        if (target >= 0 && target < a.vocab) {
            from = reinterpret_cast<const u32x4*>(static_cast<const uint8_t*>(a.H) + row * a.h_stride * elem);
            to = reinterpret_cast<u32x4*>(a.packed + (int64_t)before * row_bytes);
            if (a.twice) again = reinterpret_cast<u32x4*>(a.packed + (int64_t)(all + before) * row_bytes);
            if (threadIdx.x == 0) {
                a.index[before] = row;
                a.target[before] = (int)target;
                if (a.twice) a.target[all + before] = -1;
            }
        } else {
            if (threadIdx.x == 0) {
                a.losses[row] = 0.0f;
                if (a.logs) a.logs[row] = 0.0f;
            }
            if (a.dH) to = reinterpret_cast<u32x4*>(static_cast<uint8_t*>(a.dH) + row * a.dh_stride * elem);
        }
    } else {
        const int there = rows_of_dw(a, all), slot = there + (int)blockIdx.x - rows;
        if (slot >= (there + 255) / 256 * 256) return;
        to = reinterpret_cast<u32x4*>(a.packed + (int64_t)slot * row_bytes);
        if (threadIdx.x == 0) a.target[slot] = -1;
    }
    if (!to) return;
    for (int k = threadIdx.x; k < row_bytes / 16; k += 256) {
        const u32x4 x = from ? from[k] : u32x4{0, 0, 0, 0};
        to[k] = x;
        if (again) again[k] = x;
    }
}

// A row's maximum t and the sum of exp(z - t).  They stay apart: in L = t + log(sum) the logarithm loses the digits that t needs, and p and the loss are made of z - t, which has none of t's size.
struct RowSum {
    float top, sum;
    __device__ __forceinline__ float log_of_sum() const { return logf(sum); }
};
// What RUNS threads a row make of its pieces, each a running maximum and sum; 16 rows
template <int RUNS> struct Runs {
    float top[RUNS][17], sum[RUNS][17], plain[RUNS][17];
    // r: the row's number of the 16
    __device__ __forceinline__ void gather(const LossArgs& a, int run, int r, int row, bool there) {
        float t = -INFINITY, s = 0.0f, x = 0.0f;
        // (rows behind the last: the pieces are there, of packed zeros or of nothing yet, and nothing is made of them)
        if (there) {
#pragma unroll 4
            for (int p = run; p < a.pieces; p += RUNS) {
                const int64_t at = (int64_t)p * a.block_rows + row;
                const float of_piece = a.top[at], sum_of_piece = a.sum[at], higher = fmaxf(t, of_piece), from = higher == -INFINITY ? 0.0f : higher;
                s = s * __builtin_amdgcn_exp2f((t - from) * kLossLog2e) + sum_of_piece * __builtin_amdgcn_exp2f((of_piece - from) * kLossLog2e);
                t = higher;
                if (a.smoothing > 0.0f) x += a.plain[at];
            }
        }
        top[run][r] = t; sum[run][r] = s; plain[run][r] = x;
    }
    // `all`: the sum of z
    __device__ __forceinline__ RowSum join(int r, float& all) const {
        float t = top[0][r], s = 0.0f;
#pragma unroll 16
        for (int k = 1; k < RUNS; ++k) t = fmaxf(t, top[k][r]);
        const float from = t == -INFINITY ? 0.0f : t;
        all = 0.0f;
#pragma unroll 16
        for (int k = 0; k < RUNS; ++k) {
            s += sum[k][r] * __builtin_amdgcn_exp2f((top[k][r] - from) * kLossLog2e);
            all += plain[k][r];
        }
        return {t, s};
    }
};
// (-(1 - smoothing) z[target] - smoothing mean(z) as differences from t)
__device__ __forceinline__ void store_loss(const LossArgs& a, int row, int64_t to, const RowSum& of, float all) {
    const float log = of.log_of_sum(), L = of.top + log;
    float loss = fmaf(1.0f - a.smoothing, of.top - a.hit[row], log);
    if (a.smoothing > 0.0f) loss = fmaf(a.smoothing, of.top - all / (float)a.vocab, loss);
    if (a.z_loss > 0.0f) loss = fmaf(a.z_loss * L, L, loss);
    a.losses[to] = loss;
    if (a.logs) a.logs[to] = L;
}

// Maxima, sums and losses: 16 rows a workgroup.  (4096 rows of 250 pieces 9 us, 8192 of 1000 25.)
template <int RUNS>
__global__ __launch_bounds__(16 * RUNS) void k_loss_rows(LossArgs a, int fp16) {
    __shared__ Runs<RUNS> runs;
    const int rows = rows_of_block(a), run = threadIdx.x >> 4, r = threadIdx.x & 15, row = blockIdx.x * 16 + r;
    if ((int)blockIdx.x * 16 >= rows) return;
    runs.gather(a, run, r, row, row < rows);
    __syncthreads();
    float bound = 0.0f;
    if (run == 0 && row < rows) {
        float all;
        const RowSum of = runs.join(r, all);
        const int64_t to = a.index[a.block * a.block_rows + row];
        store_loss(a, row, to, of, all);
        if (a.train) {
            const float factor = a.weights ? a.scale * a.weights[to] : a.scale;
            a.row_top[row] = of.top;
            a.row_sum[row] = of.sum;
            a.factor[row] = factor;
            bound = fabsf(factor) * fmaf(2.0f * a.z_loss, fabsf(of.top + of.log_of_sum()), 2.0f);
        }
    }
    if (!fp16 || !a.train || run) return;
    // the largest gradient of z that there can be: 16 lanes' maximum, and an atomic one, whose order is of no matter.  (What is not finite has no say.)
    bound = bound <= 3.402823466e38f ? bound : 0.0f;
#pragma unroll
    for (int d = 8; d; d /= 2) bound = fmaxf(bound, __shfl_xor(bound, d));
    if (r == 0) atomicMax(reinterpret_cast<unsigned*>(a.count) + 1, __float_as_uint(bound));
}

constexpr int kDzRuns = 16, kDzPieces = 4 * kDzRuns;                     // threads a row, and the most pieces that k_loss_dz joins
constexpr int kDzColumns = 512;                                          // of a workgroup of k_loss_dz, in steps of 128

// dz = (p (1 + 2 z_loss L) - smoothing / vocab - (1 - smoothing) [v = target]) factor in place of the exponentials: 16 rows a workgroup, so that the pieces' maxima come in
// whole lines.  Two bytes read and two written an element: bound by memory (4096 rows of 32000 in bf16 80 us, 6.6 TB/s).  ROWS: the rows' maxima and sums are made here too, by every workgroup of a row (and the losses by the first), which
// saves a launch where the pieces are few (64 x 256 x 1000 in fp32, all of a call: 30.4 us, 32.1 with it); not in fp16, whose scale goes by all rows.
template <typename D, bool ROWS>
__global__ __launch_bounds__(256) void k_loss_dz(LossArgs a) {
    const int rows = rows_of_block(a), chunks = (a.padded + kDzColumns - 1) / kDzColumns;
    const int row = (int)(blockIdx.x / chunks) * 16 + (threadIdx.x >> 4), v0 = (int)(blockIdx.x % chunks) * kDzColumns + (threadIdx.x & 15) * 8;
    const int all_rows = rows_of_dw(a, rows);
    if ((int)(blockIdx.x / chunks) * 16 >= (all_rows + 63) / 64 * 64) return;
    typename D::elem* const e = reinterpret_cast<typename D::elem*>(a.e) + (int64_t)row * a.padded;
    const bool there = row < rows;
    RowSum of = {0.0f, 1.0f};
    float factor = 0.0f;
    if constexpr (ROWS) {
        __shared__ Runs<kDzRuns> runs;
        const int r = threadIdx.x & 15, of_r = row - (int)(threadIdx.x >> 4) + r;
        runs.gather(a, threadIdx.x >> 4, r, of_r, of_r < rows);
        __syncthreads();
        if (there) {
            float all;
            of = runs.join(threadIdx.x >> 4, all);
            const int64_t to = a.index[a.block * a.block_rows + row];
            factor = (a.weights ? a.scale * a.weights[to] : a.scale) * gradient_scale<D>(a);
            if (v0 == 0) store_loss(a, row, to, of, all);
        }
    } else if (there) {
        of = {a.row_top[row], a.row_sum[row]};
        factor = a.factor[row] * gradient_scale<D>(a);
    }
    const float log = of.log_of_sum(), share = a.smoothing / (float)a.vocab, rise = fmaf(2.0f * a.z_loss, of.top + log, 1.0f), of_sum = 1.0f / (of.sum * kLossTop<D>) * rise * factor;
    const int target = there ? a.target[row] : -1;
#pragma unroll 4
    for (int c = 0; c < kDzColumns; c += 128) {
        const int v = v0 + c;
        if (v >= a.padded) break;
        Eight x, second;
#pragma unroll
        for (int k = 0; k < 8; ++k) second.x[k] = 0.0f;
        if (there) {
            x = load_eight<LossExp<D>>(reinterpret_cast<const typename LossExp<D>::elem*>(e + v), 8);
            const float of_piece = a.top[(int64_t)(v / a.piece) * a.block_rows + row];
            const float by = __builtin_amdgcn_exp2f((of_piece - of.top) * kLossLog2e) * of_sum;
#pragma unroll
            for (int k = 0; k < 8; ++k) x.x[k] = v + k < a.vocab ? fmaf(x.x[k], by, -share * factor) : 0.0f;
            if (target >= v && target < v + 8) {
                // of the target z is there in fp32: p - 1 without what the rounding of p would leave of it
                const float p_less_1 = expm1f((a.hit[row] - of.top) - log), there_now = (p_less_1 * rise + (rise - 1.0f) + a.smoothing - share) * factor;
                const float rest = D::size == 2 ? there_now - widen<D>(narrow<D>(there_now)) : 0.0f;
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    x.x[k] = v + k == target ? there_now : x.x[k];
                    second.x[k] = v + k == target ? rest : 0.0f;
                }
                if (D::size == 2) a.left[row] = rest;
            }
        } else {
#pragma unroll
            for (int k = 0; k < 8; ++k) x.x[k] = 0.0f;
        }
        if (there || row >= all_rows) store_eight<D>(e + v, x, 8);
        if (there && a.twice) store_eight<D>(e + (int64_t)rows * a.padded + v, second, 8);
    }
}

// The parts of dH, added in their order.  (Five of 1800 rows of 1000: 8.2 us, 4.6 TB/s.)
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
    if constexpr (D::size == 2)
        sum += a.left[row] * (1.0f / gradient_scale<D>(a)) * four_of<D>(static_cast<const uint8_t*>(a.W) + (a.target[row] * a.w_stride + d) * D::size);
    store_four<D>(static_cast<uint8_t*>(a.dH) + (a.index[a.block * a.block_rows + row] * a.dh_stride + d) * D::size, sum[0], sum[1], sum[2], sum[3]);
}

// ------------------------------------------------------------------ plan
static int64_t ceil_to(int64_t x, int64_t to) { return (x + to - 1) / to * to; }

// The time of tiles of products over `length`, in us, by a rough account: operations a us of a CU whose workgroups are few in all (fewer than half the CUs: clocks are higher then), of
// one among many, and of as many as it holds; and what a round of them costs besides.  Measured with tiles of 256, 128, 64 and 32: logits of 1000 rows, width 1024, 8000 words in bf16 30, 27, 32 and 83 us;
// 64 x 1024 x 8000 26, 16, 8.4 and 7.2; 64 x 4096 x 1000 72, 45, 22 and 9.7, in fp32 (128 and less) 274, 80 and 27.  Of 80 calls of random sizes from 16 x 64 x 500 on, what it takes is 1 % behind
// the best tile of the logits on average, and 3 % behind the best tile and parts of the gradients.
struct TileRate { int tile, at_once; double few, one, all, round; };
constexpr TileRate kTileRates[7] = {{256, 1, 7.5e6, 4.8e6, 4.8e6, 5.0}, {128, 2, 3.3e6, 2.6e6, 3.6e6, 3.0}, {64, 4, 1.35e6, 1.0e6, 2.6e6, 2.0}, {32, 2, 1.4e6, 0.8e6, 1.1e6, 3.0},
                                    {128, 2, 0.49e6, 0.49e6, 0.5e6, 3.0}, {64, 4, 0.39e6, 0.39e6, 0.52e6, 2.0}, {32, 2, 0.33e6, 0.33e6, 0.38e6, 3.0}};   // the last three: fp32
static int64_t tiles_of(int64_t m, int64_t n, const TileRate& r) { return (m + r.tile - 1) / r.tile * ((n + r.tile - 1) / r.tile); }
// One of `tiles` in a launch, and all of them
static int at_once(int64_t tiles, const TileRate& r) { return (int)std::min<int64_t>(r.at_once, (tiles + 255) / 256); }
static double tile_us(int64_t tiles, int64_t length, const TileRate& r) {
    const int here = at_once(tiles, r);
    return r.round + here * 2.0 * r.tile * r.tile * (double)length / (tiles <= 128 ? r.few : std::min(here * r.one, r.all));
}
static double tiles_us(int64_t tiles, int64_t length, const TileRate& r) {
    const int in_round = 256 * at_once(tiles, r);
    return (double)((tiles + in_round - 1) / in_round) * tile_us(tiles, length, r);
}
// Tiles of two kinds in a launch, m longer ones first, each going where there is room
static double two_kinds_us(int64_t m, int64_t m_length, int64_t n, int64_t n_length, const TileRate& r) {
    const double x = tile_us(m + n, m_length, r), y = tile_us(m + n, n_length, r);
    const int slots = 256 * at_once(m + n, r);
    if (m < slots) {                                                     // the others run beside them, and what is left of the longer ones then has the CUs to itself
        const double with = (double)((n + slots - m - 1) / (slots - m)) * y, alone = m > 256 ? tile_us(m, m_length, r) : r.round + 2.0 * r.tile * r.tile * (double)m_length / r.one;
        if (with < x) return with + (1.0 - with / x) * alone;
    }
    const int64_t whole = m / slots, late = m % slots;
    const double early = (double)whole * x, then = late ? early + x : early, even = std::max(early, ((double)m * x + (double)n * y) / slots);
    const auto done = [&](double t) { return (double)(slots - late) * std::floor((t - early) / y + 1e-6) + (double)late * std::max(std::floor((t - then) / y + 1e-6), 0.0); };
    double best = 1e30;
    for (const double from : {early, then})
        for (double k = std::max(std::ceil((even - from) / y - 1e-6), 0.0);; ++k)
            if (done(from + k * y) >= (double)n) { best = std::min(best, from + k * y); break; }
    return std::max(best, then);
}

constexpr int kTwiceRows = 32;
void plan_loss(LossArgs& a, lsp_dtype dtype) {
    const bool fp32 = dtype == LSP_F32;
    const int64_t size = fp32 ? 4 : 2;
    a.padded = (int)ceil_to(a.vocab, 256);
    const int64_t row = std::max<int64_t>(a.width, a.train ? a.padded : 0) * size;
    const int64_t most = std::max<int64_t>(256, std::min<int64_t>((int64_t)kLossBytes / row, a.train ? LSP_MAX_ROWS : 16384) / 256 * 256);
    a.blocks = (int)((a.rows + most - 1) / most);
    // 16 bits: the error of dW goes by the roundings of the targets' dz, of few rows by chance.  What they take off has rows of its own where those cost nothing: a stage of dW's products has 64.
    a.twice = a.train && !fp32 && a.rows <= kTwiceRows;
    a.block_rows = (int)ceil_to(a.twice ? 2 * a.rows : (a.rows + a.blocks - 1) / a.blocks, 256);
    a.blocks = (int)((a.rows + a.block_rows - 1) / a.block_rows);
    const int64_t rows = std::min<int64_t>(a.rows, a.block_rows), dw_rows = a.twice ? 2 * rows : rows;
    double least[2] = {1e30, 1e30};
    for (int k = fp32 ? 4 : 0; k < (fp32 ? 7 : 4); ++k) {
        const TileRate& r = kTileRates[k];
        const double us = tiles_us(tiles_of(a.vocab, rows, r), a.width, r);
        if (us < least[0]) { least[0] = us; a.tile[0] = r.tile; }
        // both gradients; parts' sums are written and read again, at 5 TB/s, by a launch more
        const int64_t dh = tiles_of(a.width, rows, r), dw = tiles_of(a.width, a.vocab, r);
        for (int s = 1; s <= 32 && (s == 1 || (a.vocab / s >= 128 && dh * s <= 1024)); ++s) {
            const int64_t part = (a.vocab + s - 1) / s;
            const double back = (dw_rows > part ? two_kinds_us(dw, dw_rows, dh * s, part, r) : two_kinds_us(dh * s, part, dw, dw_rows, r)) + (s > 1 ? 4.0 + 1.6e-6 * (double)s * (double)(rows * a.width) : 0.0);
            if (back < least[1]) { least[1] = back; a.tile[1] = r.tile; a.dh_splits = s; a.dw_first = dw_rows > part; }
        }
    }
    a.piece = std::max(a.tile[0] / 2, 32);
    a.pieces = a.padded / a.piece;
    a.dh_room = (int)((rows + a.tile[1] - 1) / a.tile[1]) * a.dh_splits;
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
        take(a.row_top, (size_t)a.block_rows * 4);
        take(a.row_sum, (size_t)a.block_rows * 4);
        take(a.factor, (size_t)a.block_rows * 4);
        take(a.left, size == 2 ? (size_t)a.block_rows * 4 : 0);
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
        const bool fp16 = std::is_same<D, F16>::value, together = a.train && !fp16 && a.pieces <= kDzPieces;
        if (a.pieces > kDzPieces) hipLaunchKernelGGL(k_loss_rows<64>, dim3((unsigned)(a.block_rows / 16)), dim3(1024), 0, st, a, (int)fp16);
        else if (!together) hipLaunchKernelGGL(k_loss_rows<kDzRuns>, dim3((unsigned)(a.block_rows / 16)), dim3(16 * kDzRuns), 0, st, a, (int)fp16);
        if ((e = hipGetLastError()) != hipSuccess || !a.train) continue;
        const dim3 dz((unsigned)(a.block_rows / 16 * ((a.padded + kDzColumns - 1) / kDzColumns)));
        if constexpr (!std::is_same<D, F16>::value) {
            if (together) hipLaunchKernelGGL((k_loss_dz<D, true>), dz, dim3(256), 0, st, a);
        }
        if (!together) hipLaunchKernelGGL((k_loss_dz<D, false>), dz, dim3(256), 0, st, a);
        if ((e = hipGetLastError()) != hipSuccess) break;
        if ((e = launch_loss_back<D>(a, st)) != hipSuccess) break;
        if (a.dH && a.dh_splits > 1) {
            hipLaunchKernelGGL(k_loss_dh_sum<D>, dim3((unsigned)(((int64_t)a.block_rows * (a.width / 4) + 255) / 256)), dim3(256), 0, st, a);
            e = hipGetLastError();
        }
    }
    return e;
}

hipError_t launch_loss(LossArgs& a, lsp_dtype dtype, hipStream_t st) {
    return dtype == LSP_F32 ? launch_blocks<F32>(a, dtype, st) : dtype == LSP_F16 ? launch_blocks<F16>(a, dtype, st) : launch_blocks<BF16>(a, dtype, st);
}

}  // namespace lsp

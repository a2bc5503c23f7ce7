// Tiles of a matrix product C[m][n] = sum_k A[m][k] B[n][k] on the matrix cores, for the kernels that do something with C before it is stored.
//
// Either operand may have k along its rows in memory or across them; both come straight into LDS as they lie there (Tile in attention.h says how), and an operand
// whose k runs across the rows is transposed by the reads that make fragments of it.  K goes by in steps of 128 bytes of an operand with k along its rows; two
// buffers, filled in turn: while a step is multiplied the next one is on its way.  A wave holds MI x NI products of 32 x 32: accumulators [n block][m block], so
// that a lane has for one n four m that follow one another.
#pragma once

#include "attention.h"

namespace lsp {

// One operand of a product: element (row, column) at first + row * row_bytes + column elements.  ACROSS: k counts rows, otherwise columns.
struct Operand { const uint8_t* first; int64_t row_bytes; };

#if defined(__HIPCC__)
// N rows (or columns, where ACROSS) by BK of k.
template <typename D, int N, int BK, int WAVES, bool ACROSS> struct OperandTile {
    using T = Tile<D, ACROSS ? N : BK>;
    static constexpr int kRows = ACROSS ? BK : N;
    static constexpr uint32_t kBytes = (uint32_t)N * BK * D::size;
    static constexpr int kLoads = kBytes / 1024, kCount = (kLoads + WAVES - 1) / WAVES;
    static_assert(kBytes % 1024 == 0 && kLoads % WAVES == 0, "whole loads for every wave");
    uint32_t off[kCount];
    int      k[kCount];                               // of the step's k that this load has
    uint32_t row_at[2], column_at[2];

    // `there`: how many of the N there are
    __device__ __forceinline__ void setup(int64_t row_bytes, int there, int wave, int lane) {
#pragma unroll
        for (int i = 0; i < kCount; ++i) {
            uint32_t r, unit;
            T::at_place((i * WAVES + wave) * 64 + lane, r, unit);
            const int column = (int)unit * T::kUnitElems;
            k[i] = ACROSS ? (int)r : column;
            off[i] = (ACROSS ? column : (int)r) < there ? r * (uint32_t)row_bytes + unit * 16u : kNowhere;
        }
        const uint32_t row = lane & 31, h = (uint32_t)lane >> 5;
#pragma unroll
        for (int x = 0; x < 2; ++x) {
            if constexpr (D::size == 2) {
                row_at[x] = T::place(row, 2 * x + h);
                column_at[x] = T::place(8 * h + 4 * x + ((lane >> 2) & 3), ((lane >> 4) & 1) * 2 + ((lane & 3) >> 1)) + (lane & 1) * 8u;
            } else {
                row_at[x] = T::place(row, 2 * h + x);
                column_at[x] = T::place(8 * h + 4 * x, (lane & 31) >> 2) + (lane & 3) * 4u;
            }
        }
    }
    // The step that begins at `first` and has `left` of k
    __device__ __forceinline__ void fetch(const uint8_t* first, int left, Lds tile, int wave) const {
        const Buffer b = buffer_from(first);
#pragma unroll
        for (int i = 0; i < kCount; ++i)
            __builtin_amdgcn_raw_ptr_buffer_load_lds(b, (LSP_SHARED_AS void*)(tile + (i * WAVES + wave) * 1024u), 16, (int)(k[i] < left ? off[i] : kNowhere), 0, 0, 0);
    }
    // Rows (columns) 32 block + 0..31, k = 16 ks + 8 h + 0..7 for the lane's half h
    __device__ __forceinline__ Frag<D> frag(Lds tile, int block, int ks) const {
        Frag<D> f;
        if constexpr (!ACROSS) {
            const Lds t = tile + block * (32 / 4 * T::kUnits * 64);
            if constexpr (D::size == 2) f.w = lds_read<u32x4>(t + row_at[ks & 1] + (ks >> 1) * 256);
            else {
                const f32x4 a = lds_read<f32x4>(t + row_at[0] + ks * 256), b = lds_read<f32x4>(t + row_at[1] + ks * 256);
#pragma unroll
                for (int j = 0; j < 4; ++j) { f.w[j] = a[j]; f.w[4 + j] = b[j]; }
            }
        } else {
            const Lds t = tile + ks * (16 / 4 * T::kUnits * 64) + block * (D::size * 128);
            if constexpr (D::size == 2) {
#pragma unroll
                for (int x = 0; x < 2; ++x) {
                    const s16x4 v = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LSP_SHARED_AS s16x4*)(t + column_at[x]));
                    u32x2 u;
                    __builtin_memcpy(&u, &v, 8);
                    f.w[2 * x] = u[0]; f.w[2 * x + 1] = u[1];
                }
            } else {
#pragma unroll
                for (int j = 0; j < 8; ++j) f.w[j] = lds_read<float>(t + column_at[j >> 2] + (j & 3) * 64);
            }
        }
        return f;
    }
};

template <typename D, int BM_, int BN_, int WM_, int WN_, bool A_ACROSS, bool B_ACROSS> struct Product {
    static constexpr int BM = BM_, BN = BN_, WM = WM_, WN = WN_, BK = 128 / D::size, kWaves = WM * WN, kThreads = 64 * kWaves, MI = BM / WM / 32, NI = BN / WN / 32, kSteps = BK / 16;
    using A = OperandTile<D, BM, BK, kWaves, A_ACROSS>;
    using B = OperandTile<D, BN, BK, kWaves, B_ACROSS>;
    static constexpr uint32_t kStage = A::kBytes + B::kBytes;
    static constexpr uint32_t kLds = 2 * kStage;

    f32x16 acc[NI][MI];

    __device__ __forceinline__ void step(const A& a, const B& b, Lds __restrict from, int wm, int wn) {
#pragma unroll
        for (int ks = 0; ks < kSteps; ++ks) {
            Frag<D> x[MI], y[NI];
#pragma unroll
            for (int i = 0; i < MI; ++i) x[i] = a.frag(from, wm * MI + i, ks);
#pragma unroll
            for (int j = 0; j < NI; ++j) y[j] = b.frag(from + A::kBytes, wn * NI + j, ks);
#pragma unroll
            for (int j = 0; j < NI; ++j)
#pragma unroll
                for (int i = 0; i < MI; ++i) acc[j][i] = mma<D>(x[i], y[j], acc[j][i]);
        }
    }
    // k from 0 to `length`; m_there, n_there: how many rows (columns) of the tile there are.  All waves are done with LDS when it returns.
    __device__ __forceinline__ void run(const Operand& oa, const Operand& ob, int64_t length, int m_there, int n_there, Lds lds) {
        const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, wm = wave % WM, wn = wave / WM;
        A a;
        B b;
        a.setup(oa.row_bytes, m_there, wave, lane);
        b.setup(ob.row_bytes, n_there, wave, lane);
#pragma unroll
        for (int j = 0; j < NI; ++j)
#pragma unroll
            for (int i = 0; i < MI; ++i) acc[j][i] = zeros16();
        const int64_t a_step = A_ACROSS ? oa.row_bytes * BK : BK * D::size, b_step = B_ACROSS ? ob.row_bytes * BK : BK * D::size;
        const uint8_t* pa = oa.first;
        const uint8_t* pb = ob.first;
        int64_t left = length;
        const auto fetch = [&](Lds into) {
            const int n = (int)min(left, (int64_t)BK);
            a.fetch(pa, n, into, wave);
            b.fetch(pb, n, into + A::kBytes, wave);
            pa += a_step; pb += b_step; left -= BK;
        };
        if (left > 0) fetch(lds);
        for (int64_t k = 0; k < length; k += 2 * BK) {
            arrived_for_all();
            if (left > 0) fetch(lds + kStage);
            step(a, b, lds, wm, wn);
            if (k + BK >= length) break;
            arrived_for_all();
            if (left > 0) fetch(lds);
            step(a, b, lds + kStage, wm, wn);
        }
        __syncthreads();
    }
};

// Tile `item` of tiles_m x tiles_n, in panels of a few n so that the workgroups of an XCD, which get items that follow one another, read few rows of both operands
__device__ __forceinline__ void tile_of_item(uint32_t item, uint32_t tiles_m, uint32_t tiles_n, uint32_t& m, uint32_t& n) {
    constexpr uint32_t kPanel = 4;
    const uint32_t panel = item / (kPanel * tiles_m), inside = item - panel * kPanel * tiles_m, width = min(kPanel, tiles_n - panel * kPanel);
    m = inside / width;
    n = panel * kPanel + inside % width;
}
// Which of `items` workgroup `block` does, or `items`: none.  Workgroups go round the eight XCDs; each XCD gets a run of items.
__device__ __forceinline__ uint32_t item_of_block(uint32_t block, uint32_t items) {
    const uint32_t xcd = block & 7u, nth = block >> 3, share = items >> 3, rest = items & 7u;
    return nth < share + (xcd < rest ? 1u : 0u) ? xcd * share + min(xcd, rest) + nth : items;
}
#endif

}  // namespace lsp

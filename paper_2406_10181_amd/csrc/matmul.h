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
    uint32_t at[2];                                   // where this lane reads: see frag()

    // Which k of a step load i has
    __device__ __forceinline__ static int k_of(int i, int wave, int lane) {
        uint32_t r, unit;
        T::at_place((i * WAVES + wave) * 64 + lane, r, unit);
        return ACROSS ? (int)r : (int)unit * T::kUnitElems;
    }
    // `there`: how many of the N there are
    __device__ __forceinline__ void setup(int64_t row_bytes, int there, int wave, int lane) {
#pragma unroll
        for (int i = 0; i < kCount; ++i) {
            uint32_t r, unit;
            T::at_place((i * WAVES + wave) * 64 + lane, r, unit);
            off[i] = (ACROSS ? (int)unit * T::kUnitElems : (int)r) < there ? r * (uint32_t)row_bytes + unit * 16u : kNowhere;
        }
        const uint32_t row = lane & 31, h = (uint32_t)lane >> 5;
#pragma unroll
        for (int x = 0; x < 2; ++x) {
            if constexpr (D::size == 2)
                at[x] = ACROSS ? T::place(8 * h + 4 * x + ((lane >> 2) & 3), ((lane >> 4) & 1) * 2 + ((lane & 3) >> 1)) + (lane & 1) * 8u : T::place(row, 2 * x + h);
            else
                at[x] = ACROSS ? T::place(8 * h + 4 * x, (lane & 31) >> 2) + (lane & 3) * 4u : T::place(row, 2 * h + x);
        }
    }
    // The step that begins at `first`; PART: only `left` of its k are there
    template <bool PART> __device__ __forceinline__ void fetch(const uint8_t* first, int left, Lds tile, int wave, int lane) const {
        const Buffer b = buffer_from(first);
#pragma unroll
        for (int i = 0; i < kCount; ++i) {
            const uint32_t o = PART && k_of(i, wave, lane) >= left ? kNowhere : off[i];
            __builtin_amdgcn_raw_ptr_buffer_load_lds(b, (LSP_SHARED_AS void*)(tile + (i * WAVES + wave) * 1024u), 16, (int)o, 0, 0, 0);
        }
    }
    // Rows (columns) 32 block + 0..31, k = 16 ks + 8 h + 0..7 for the lane's half h
    __device__ __forceinline__ Frag<D> frag(Lds tile, int block, int ks) const {
        Frag<D> f;
        if constexpr (!ACROSS) {
            const Lds t = tile + block * (32 / 4 * T::kUnits * 64);
            if constexpr (D::size == 2) f.w = lds_read<u32x4>(t + at[ks & 1] + (ks >> 1) * 256);
            else {
                const f32x4 a = lds_read<f32x4>(t + at[0] + ks * 256), b = lds_read<f32x4>(t + at[1] + ks * 256);
#pragma unroll
                for (int j = 0; j < 4; ++j) { f.w[j] = a[j]; f.w[4 + j] = b[j]; }
            }
        } else {
            const Lds t = tile + ks * (16 / 4 * T::kUnits * 64) + block * (D::size * 128);
            if constexpr (D::size == 2) {
#pragma unroll
                for (int x = 0; x < 2; ++x) {
                    const s16x4 v = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LSP_SHARED_AS s16x4*)(t + at[x]));
                    u32x2 u;
                    __builtin_memcpy(&u, &v, 8);
                    f.w[2 * x] = u[0]; f.w[2 * x + 1] = u[1];
                }
            } else {
#pragma unroll
                for (int j = 0; j < 8; ++j) f.w[j] = lds_read<float>(t + at[j >> 2] + (j & 3) * 64);
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

    struct Frags { Frag<D> x[MI], y[NI]; };
    __device__ __forceinline__ static void read(Frags& f, const A& a, const B& b, Lds from, int wm, int wn, int ks) {
#pragma unroll
        for (int i = 0; i < MI; ++i) f.x[i] = a.frag(from, wm * MI + i, ks);
#pragma unroll
        for (int j = 0; j < NI; ++j) f.y[j] = b.frag(from + A::kBytes, wn * NI + j, ks);
    }
    // One step: while `from` is multiplied, `into` is filled.  The fragments of 16 k are read while those before are multiplied, and no further ahead: with the reads of a whole step
    // ahead the accumulators would not stay in registers.
    template <typename Fill> __device__ __forceinline__ void step(const A& a, const B& b, Lds __restrict from, Lds __restrict into, int wm, int wn, Fill&& fill) {
        fill(into);
        Frags f[2];
        read(f[0], a, b, from, wm, wn, 0);
#pragma unroll
        for (int ks = 0; ks < kSteps; ++ks) {
            __builtin_amdgcn_sched_barrier(0);
            if (ks + 1 < kSteps) read(f[(ks + 1) & 1], a, b, from, wm, wn, ks + 1);
#pragma unroll
            for (int j = 0; j < NI; ++j)
#pragma unroll
                for (int i = 0; i < MI; ++i) acc[j][i] = mma<D>(f[ks & 1].x[i], f[ks & 1].y[j], acc[j][i]);
        }
    }
    // k from 0 to `length`; m_there, n_there: how many rows (columns) of the tile there are.  All waves are done with LDS when it returns.
    __device__ __forceinline__ void run(const Operand& oa, const Operand& ob, int length, int m_there, int n_there, Lds lds) {
        const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, wm = wave % WM, wn = wave / WM;
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
        int left = length;
        const auto fetch = [&](Lds into) {
            if (left >= BK) {
                a.template fetch<false>(pa, left, into, wave, lane);
                b.template fetch<false>(pb, left, into + A::kBytes, wave, lane);
            } else if (left > 0) {
                a.template fetch<true>(pa, left, into, wave, lane);
                b.template fetch<true>(pb, left, into + A::kBytes, wave, lane);
            }
            pa += a_step; pb += b_step; left -= BK;
        };
        fetch(lds);
        const int steps = (length + BK - 1) / BK;
        for (int t = 0; t < steps; ++t) {
            const uint32_t now = (t & 1) * kStage;
            arrived_for_all();
            step(a, b, lds + now, lds + (kStage - now), wm, wn, fetch);
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

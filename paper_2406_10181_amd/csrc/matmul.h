// Tiles of a matrix product C[m][n] = sum_k A[m][k] B[n][k] on the matrix cores, for the kernels that do something with C before it is stored.
//
// Either operand may have k along its rows in memory or across them; both come straight into LDS as they lie there (Tile in attention.h says how), and an operand
// whose k runs across the rows is transposed by the reads that make fragments of it.  K goes by in stages of 128 bytes of an operand with k along its rows.
//
// The products are of 16 x 16 tiles, 32 values of k at a time (v_mfma_f32_16x16x32 in 16 bits, eight v_mfma_f32_16x16x4 in fp32): lane l supplies A[l % 16][8 (l / 16) + 0..7]
// and B alike, and holds C[4 (l / 16) + i][l % 16] in accumulator register i.  32 x 32 tiles would read LDS no less, and what a product with random numbers reaches is a matter of the power
// that it takes: products of registers alone, in bf16, 2047 TFLOP/s with 16 x 16 x 32 and 1753 with 32 x 32 x 16 (of zeros 2400 and 2345).
// A wave holds MI x NI of them, accumulators [n block][m block], so that a lane has for one n four m that follow one another.
#pragma once

#include "attention.h"
#include "rows.h"

namespace lsp {

// One operand of a product: element (row, column) at first + row * row_bytes + column elements.  ACROSS: k counts rows, otherwise columns.
struct Operand { const uint8_t* first; int64_t row_bytes; };

#if defined(__HIPCC__)
template <typename D> __device__ __forceinline__ f32x4 mma16(const Frag<D>& a, const Frag<D>& b, f32x4 c) {
    if constexpr (std::is_same<D, BF16>::value) {
        bf16x8 x, y;
        __builtin_memcpy(&x, &a.w, 16); __builtin_memcpy(&y, &b.w, 16);
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(x, y, c, 0, 0, 0);
    } else if constexpr (std::is_same<D, F16>::value) {
        f16x8 x, y;
        __builtin_memcpy(&x, &a.w, 16); __builtin_memcpy(&y, &b.w, 16);
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(x, y, c, 0, 0, 0);
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a.w[j], b.w[j], c, 0, 0, 0);
        return c;
    }
}

// The larger, and the sum, of the values of the four lanes that share a column of C (l, l ^ 16, l ^ 32, l ^ 48), in all of them
__device__ __forceinline__ float quarters_max(float x) {
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return halves_max(fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1])));
}
__device__ __forceinline__ float quarters_sum(float x) {
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return halves_sum(__uint_as_float(r[0]) + __uint_as_float(r[1]));
}

// N rows (or columns, where ACROSS) by BK of k.
template <typename D, int N, int BK, int WAVES, bool ACROSS> struct OperandTile {
    using T = Tile<D, ACROSS ? N : BK>;
    static constexpr uint32_t kBytes = (uint32_t)N * BK * D::size;
    static constexpr int kLoads = kBytes / 1024, kCount = (kLoads + WAVES - 1) / WAVES;
    static_assert(kBytes % 1024 == 0 && kLoads % WAVES == 0, "whole loads for every wave");
    static constexpr uint32_t kRows4 = T::kUnits * 64;  // bytes of four rows
    uint32_t off[kCount];
    uint32_t at[2][2];                                // where this lane reads: see frag()

    // Which k of a stage load i has
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
        const uint32_t row = lane & 15, g = (uint32_t)lane >> 4;
#pragma unroll
        for (int x = 0; x < 2; ++x)
#pragma unroll
            for (int p = 0; p < 2; ++p) {
                if constexpr (D::size == 2)
                    at[x][p] = ACROSS ? T::place(8 * g + 4 * x + ((lane >> 2) & 3), 2 * p + ((lane & 3) >> 1)) + (lane & 1) * 8u : T::place(row, g);
                else
                    at[x][p] = ACROSS ? T::place(8 * g + 4 * x, row >> 2) + (lane & 3) * 4u : T::place(row, 2 * g + x);
            }
    }
    // Load i of the stage that begins at `first`; PART: only `left` of its k are there
    template <bool PART> __device__ __forceinline__ void fetch(const uint8_t* first, int left, int i, Lds tile, int wave, int lane) const {
        const uint32_t o = PART && k_of(i, wave, lane) >= left ? kNowhere : off[i];
        __builtin_amdgcn_raw_ptr_buffer_load_lds(buffer_from(first), (LSP_SHARED_AS void*)(tile + (i * WAVES + wave) * 1024u), 16, (int)o, 0, 0, 0);
    }
    // Rows (columns) 16 block + 0..15, k = 32 ks + 0..31.  Across: the transposing read takes four rows of 16 columns from 16 lanes and gives each lane one column of them.
    __device__ __forceinline__ Frag<D> frag(Lds tile, int block, int ks) const {
        Frag<D> f;
        if constexpr (!ACROSS) {
            const Lds t = tile + block * (4 * kRows4);
            if constexpr (D::size == 2) f.w = lds_read<u32x4>(t + at[0][0] + ks * 256);
            else {
                const f32x4 a = lds_read<f32x4>(t + at[0][0]), b = lds_read<f32x4>(t + at[1][0]);
#pragma unroll
                for (int j = 0; j < 4; ++j) { f.w[j] = a[j]; f.w[4 + j] = b[j]; }
            }
        } else if constexpr (D::size == 2) {
            const Lds t = tile + ks * (8 * kRows4) + (block >> 1) * 256;
#pragma unroll
            for (int x = 0; x < 2; ++x) {
                const s16x4 v = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LSP_SHARED_AS s16x4*)(t + at[x][block & 1]));
                u32x2 u;
                __builtin_memcpy(&u, &v, 8);
                f.w[2 * x] = u[0]; f.w[2 * x + 1] = u[1];
            }
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) f.w[j] = lds_read<float>(tile + block * 256 + at[j >> 2][0] + (j & 3) * 64);
        }
        return f;
    }
};

// GROUPS of waves, each with buffers of its own, take the stages of a tile by turns, and the first adds up what they have: for tiles that are few.  A stage of a wave with 2 x 2 small tiles is a chain of
// two reads of LDS, two times four products and a barrier, 0.3 us whatever is on its way; deeper buffers do not shorten it.
template <typename D, int BM_, int BN_, int WM_, int WN_, bool A_ACROSS, bool B_ACROSS, int GROUPS = 1> struct Product {
    static constexpr int BM = BM_, BN = BN_, WM = WM_, WN = WN_, BK = 128 / D::size, kWaves = WM * WN, kThreads = 64 * kWaves * GROUPS, MI = BM / WM / 16, NI = BN / WN / 16, kSteps = BK / 32;
    static constexpr int kRange = 16 * MI;            // m of a wave
    using A = OperandTile<D, BM, BK, kWaves, A_ACROSS>;
    using B = OperandTile<D, BN, BK, kWaves, B_ACROSS>;
    // Three buffers for A and two for B: 160 KiB for 256 x 256 in 16 bits, all that a CU has
    static constexpr uint32_t kBase = 3 * A::kBytes, kOfGroup = kBase + 2 * B::kBytes, kLds = GROUPS * kOfGroup;
    static constexpr uint32_t kStored = kWaves * 32 * kRange * 4, kParts = NI * MI * 1024;  // bytes that the first group stores results through, and of a wave's results
    static_assert(GROUPS == 1 || kStored + (GROUPS - 1) * kWaves * kParts <= kLds, "room for the groups' results");
    static constexpr int kEarly = MI < 4 ? 1 : MI / 4;
    static_assert(NI % 2 == 0 && MI >= 2, "pairs of n blocks are stored, and a block of m is left when the others wait");

    f32x4 acc[NI][MI];
    Frag<D> x[MI], y[2][NI];

    // All waves have their fragments in registers, and all loads but the last LEFT of each wave have arrived.
    template <int LEFT> __device__ __forceinline__ static void arrived_but() {
        __builtin_amdgcn_sched_barrier(0);
        asm volatile("" ::: "memory");
        __builtin_amdgcn_s_waitcnt(0x0070 | (LEFT & 15) | (LEFT >> 4) << 14);       // vmcnt(LEFT), lgkmcnt(0)
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        __builtin_amdgcn_sched_barrier(0);
    }
    // One stage, whose first fragments are in registers already.  Four products on, a block of m has been multiplied and its fragment's registers take the one that
    // comes 32 k later; the fragments of n have two sets.  A little into the last 32 k everything of the stage is in registers, in all waves, and the next stage has arrived: from there on
    // the stage's buffers are filled again, and the fragments are the next stage's.
    template <bool PART> __device__ __forceinline__ void stage(const A& a, const B& b, Lds __restrict now_a, Lds __restrict now_b, Lds __restrict next_a, Lds __restrict next_b, int wm, int wn,
                                                               const uint8_t* pa, const uint8_t* pb, int left_a, int left_b, int wave, int lane) {
        constexpr int kFetches = A::kCount + B::kCount, kLate = MI - kEarly;
#pragma unroll
        for (int ks = 0; ks < kSteps; ++ks) {
            const bool last = ks + 1 == kSteps;
            const int cur = ks & 1;
#pragma unroll
            for (int i = 0; i < MI; ++i) {
#pragma unroll
                for (int j = 0; j < NI; ++j) acc[j][i] = mma16<D>(x[i], y[cur][j], acc[j][i]);
                __builtin_amdgcn_sched_barrier(0);
                if (!last) {
                    x[i] = a.frag(now_a, wm * MI + i, ks + 1);
#pragma unroll
                    for (int j = i * NI / MI; j < (i + 1) * NI / MI; ++j) y[cur ^ 1][j] = b.frag(now_b, wn * NI + j, ks + 1);
                } else if (i + 1 == kEarly) arrived_but<A::kCount>();
                else if (i >= kEarly) {
                    const int q = i - kEarly;
#pragma unroll
                    for (int j = q * NI / kLate; j < (q + 1) * NI / kLate; ++j) y[cur ^ 1][j] = b.frag(next_b, wn * NI + j, 0);
                    x[q] = a.frag(next_a, wm * MI + q, 0);
                    if (q + 1 == kLate) {
#pragma unroll
                        for (int r = kLate; r < MI; ++r) x[r] = a.frag(next_a, wm * MI + r, 0);
                    }
#pragma unroll
                    for (int l = q * kFetches / kLate; l < (q + 1) * kFetches / kLate; ++l) {
                        if (l < B::kCount) b.template fetch<PART>(pb, left_b, l, now_b, wave, lane);
                        else a.template fetch<PART>(pa, left_a, l - B::kCount, now_a, wave, lane);
                    }
                }
            }
        }
        if constexpr (kSteps % 2) {
#pragma unroll
            for (int j = 0; j < NI; ++j) y[0][j] = y[1][j];
        }
    }
    // k from 0 to `length`; m_there, n_there: how many rows (columns) of the tile there are.  All waves are done with LDS when it returns, and those of the first group have the results: false for others.
    __device__ __forceinline__ bool run(const Operand& oa, const Operand& ob, int length, int m_there, int n_there, Lds lds) {
        const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) % kWaves, group = GROUPS == 1 ? 0 : __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) / kWaves;
        const int lane = threadIdx.x & 63, wm = wave % WM, wn = wave / WM;
        const Lds whole_lds = lds;
        lds += group * kOfGroup;
        A a;
        B b;
        a.setup(oa.row_bytes, m_there, wave, lane);
        b.setup(ob.row_bytes, n_there, wave, lane);
#pragma unroll
        for (int j = 0; j < NI; ++j)
#pragma unroll
            for (int i = 0; i < MI; ++i) acc[j][i] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
        const int64_t a_step = A_ACROSS ? oa.row_bytes * BK : BK * D::size, b_step = B_ACROSS ? ob.row_bytes * BK : BK * D::size;
        const uint8_t* pa = oa.first + group * a_step;
        const uint8_t* pb = ob.first + group * b_step;
        int left_a = length - group * BK, left_b = left_a;
        const auto next_of_a = [&] { pa += GROUPS * a_step; left_a -= GROUPS * BK; };
        const auto next_of_b = [&] { pb += GROUPS * b_step; left_b -= GROUPS * BK; };
        // (behind the end too: what is loaded from nowhere is zeros, and the loads on their way are always as many)
        const auto fetch_a = [&](Lds into) {
#pragma unroll
            for (int l = 0; l < A::kCount; ++l) a.template fetch<true>(pa, left_a, l, into, wave, lane);
            next_of_a();
        };
        const auto fetch_b = [&](Lds into) {
#pragma unroll
            for (int l = 0; l < B::kCount; ++l) b.template fetch<true>(pb, left_b, l, into, wave, lane);
            next_of_b();
        };
        // A is asked for three stages ahead and B two: the 64 KiB of a stage take the CU's loads some 1500 cycles and their latency, as long as its products.
        fetch_a(lds); fetch_b(lds + kBase);
        fetch_a(lds + A::kBytes); fetch_b(lds + kBase + B::kBytes);
        fetch_a(lds + 2 * A::kBytes);
        arrived_but<2 * A::kCount + B::kCount>();
#pragma unroll
        for (int j = 0; j < NI; ++j) y[0][j] = b.frag(lds + kBase, wn * NI + j, 0);
#pragma unroll
        for (int i = 0; i < MI; ++i) x[i] = a.frag(lds, wm * MI + i, 0);
        uint32_t at_a = 0, at_b = kBase;
        const auto one = [&](auto part) {
            const uint32_t next_a = at_a == 2 * A::kBytes ? 0 : at_a + A::kBytes, next_b = 2 * kBase + B::kBytes - at_b;
            stage<decltype(part)::value>(a, b, lds + at_a, lds + at_b, lds + next_a, lds + next_b, wm, wn, pa, pb, left_a, left_b, wave, lane);
            next_of_a(); next_of_b();
            at_a = next_a; at_b = next_b;
        };
        const int stages = (length + GROUPS * BK - 1) / (GROUPS * BK), whole = length / (GROUPS * BK) - 3;   // (what stage t asks for is of stages t + 2 and t + 3)
        int t = 0;
        for (; t < whole; ++t) one(std::false_type{});
        for (; t < stages; ++t) one(std::true_type{});
        arrived_for_all();
        if constexpr (GROUPS > 1) {
            const Lds parts = whole_lds + kStored + wave * kParts + lane * 16;
            if (group) {
#pragma unroll
                for (int j = 0; j < NI; ++j)
#pragma unroll
                    for (int i = 0; i < MI; ++i) lds_write<f32x4>(parts + (group - 1) * (kWaves * kParts) + (j * MI + i) * 1024, acc[j][i]);
            }
            arrived_for_all();
            if (group) return false;
#pragma unroll
            for (int g = 0; g < GROUPS - 1; ++g)
#pragma unroll
                for (int j = 0; j < NI; ++j)
#pragma unroll
                    for (int i = 0; i < MI; ++i) acc[j][i] += lds_read<f32x4>(parts + g * (kWaves * kParts) + (j * MI + i) * 1024);
        }
        return true;
    }
};

// A wave's results of two n blocks, v[0] and v[1], as 32 rows of kRange elements: through LDS of the wave's own, so that stores are of whole lines.  `row(r)`: where row r of the 32 goes, or NULL;
// `left`: how many of the elements there are.
template <typename D, int MI, typename Row> __device__ __forceinline__ void store_two_blocks(const f32x4 (*v)[MI], float factor, Lds own, int left, int lane, Row&& row) {
    using T = Tile<D, 16 * MI>;
    const uint32_t g = (uint32_t)lane >> 4;
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        const uint32_t mine = 16 * j + (lane & 15);
#pragma unroll
        for (int i = 0; i < MI; ++i) {
            const float a = v[j][i][0] * factor, b = v[j][i][1] * factor, c = v[j][i][2] * factor, d = v[j][i][3] * factor;
            if constexpr (D::size == 4) lds_write<f32x4>(own + T::place(mine, 4 * i + g), f32x4{a, b, c, d});
            else {
                u32x2 w;
                w[0] = narrow_two<D>(a, b);
                w[1] = narrow_two<D>(c, d);
                lds_write<u32x2>(own + T::place(mine, 2 * i + (g >> 1)) + (g & 1) * 8u, w);
            }
        }
    }
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
#pragma unroll
    for (int i = 0; i < T::kUnits / 2; ++i) {
        uint32_t r, unit;
        T::at_place(i * 64 + lane, r, unit);
        const u32x4 w = lds_read<u32x4>(own + (i * 64 + lane) * 16);
        uint8_t* p = row(r);
        if (p && (int)unit * T::kUnitElems < left) *reinterpret_cast<u32x4*>(p + unit * 16u) = w;
    }
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
}

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

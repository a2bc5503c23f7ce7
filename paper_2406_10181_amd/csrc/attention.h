// Arguments of the attention kernels, and the pieces they share: fragments of the matrix instructions and tiles in LDS.
//
// Everything is built on products of 32 x 32 tiles, C[m][n] += sum_k A[m][k] B[k][n], 16 values of k at a time
// (v_mfma_f32_32x32x16 in 16 bits, eight v_mfma_f32_32x32x2 in fp32): lane l supplies eight A[l % 32][.] and eight B[.][l % 32],
// and holds C[8 (i / 4) + 4 (l / 32) + i % 4][l % 32] in accumulator register i.  Which eight values of k a lane has is free as long
// as A and B agree, and that is what joins one product to the next without moving anything between lanes: the lane's eight
// registers 8 x .. 8 x + 7 of C are rows 16 x + {4 h + 0..3, 8 + 4 h + 0..3} (h = l / 32) of column l % 32, which is a B operand whose
// k runs over these 16 rows; the A operand that meets it is read from LDS in the same order of k.  So the probabilities go from
// the accumulators of one product into the operand of the next after nothing but a rounding.
#pragma once

#include "philox.h"

namespace lsp {

struct Strided { const void* p; int64_t batch, position, head; };      // strides in elements

struct AttentionArgs {
    Strided q, k, v, o, d_o, dq, dk, dv;
    float*         L;                // [batch][heads][q_len]
    float*         delta;            // [batch][heads][q_len]: dO . O; in the backward pass
    float*         norms;            // fp16 backward: [2][kNormSlots], squares of the largest norm of a row of dO and of V that a workgroup met
    float*         partial;          // forward with several splits: O of each, then (largest score, sum) of each row; backward: parts of dK, of dV, of dQ
    const int32_t* q_lens;
    const int32_t* k_lens;
    int32_t batch, heads, kv_heads, group, q_len, k_len, head_dim, causal;
    int32_t waves;                   // of a forward workgroup: 4 or 8, each with 32 rows
    int32_t tiles;                   // row tiles of a head (or of a key head, where its query heads share the tiles)
    int32_t rows;                    // rows of a head: q_len, or group * q_len where `packed`
    int32_t packed;                  // rows are (query head of the group, query): few queries, all heads of a key head in one tile
    int32_t few;                     // forward: at most 32 rows, the kernel for these
    int32_t splits, split_tiles;     // forward: parts of the keys (at most 64), tiles of keys in each
    int32_t norm_slots;              // fp16 backward: slots in use
    int32_t key_parts, query_parts;  // backward: workgroups that share 128 keys (parts of their queries), and 128 queries (parts of their keys)
    float   scale, scale_log2;       // scale_log2 = scale * log2(e): probabilities are powers of two
    Dropout drop;
};

hipError_t launch_attention_forward(const AttentionArgs& a, lsp_dtype dtype, hipStream_t st);
hipError_t launch_attention_backward(const AttentionArgs& a, lsp_dtype dtype, hipStream_t st);
// Splits of the keys in the forward pass and what that needs; fills the tiling fields of `a`.
void plan_attention_forward(AttentionArgs& a, lsp_dtype dtype);
size_t attention_partial_bytes(const AttentionArgs& a);
void plan_attention_backward(AttentionArgs& a, lsp_dtype dtype);
size_t attention_backward_partial_bytes(const AttentionArgs& a);

constexpr int kWaveRows = 32;        // query rows (or keys, where dK and dV are made) of a wave
constexpr int kBackwardRows = 4 * kWaveRows;
constexpr int kNormSlots = 1024;

// Keys (forward, dQ) or queries (dK, dV) of a tile in LDS
template <typename D> constexpr int tile_rows() { return D::size == 2 ? 64 : 32; }
constexpr int tile_rows_of(lsp_dtype t) { return t == LSP_F32 ? 32 : 64; }

#if defined(__HIPCC__)
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef float f32x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
#define LSP_SHARED_AS __attribute__((address_space(3)))

// Forward: the running maximum stays until a new one is larger by more than 2^kLagLog2, and its own probability counts as 2^kTopLog2, in the operands as in their sums, so that
// the factor leaves with the division and only L has to take it back.  fp16 has normal numbers down to 2^-14 only: with 2^11 at the top probabilities keep all their digits down to
// 2^-25 of the largest and some down to 2^-35, and with a lag of 2^4 none is above 2^15.  (With 1 at the top one of 2^-23 was up to a quarter off, and where one key has nearly all the
// weight and no value the others' are all there is.)  bf16 and fp32 have the range.
template <typename D> constexpr float kTopLog2 = std::is_same<D, F16>::value ? 11.0f : 0.0f;
template <typename D> constexpr float kTop = std::is_same<D, F16>::value ? 2048.0f : 1.0f;
template <typename D> constexpr float kLagLog2 = std::is_same<D, F16>::value ? 4.0f : 8.0f;

// Eight values of k of one lane
template <typename D> struct Frag { u32x4 w; };
template <> struct Frag<F32> { f32x8 w; };

template <typename D> __device__ __forceinline__ f32x16 mma(const Frag<D>& a, const Frag<D>& b, f32x16 c) {
    if constexpr (std::is_same<D, BF16>::value) {
        bf16x8 x, y;
        __builtin_memcpy(&x, &a.w, 16); __builtin_memcpy(&y, &b.w, 16);
        return __builtin_amdgcn_mfma_f32_32x32x16_bf16(x, y, c, 0, 0, 0);
    } else if constexpr (std::is_same<D, F16>::value) {
        f16x8 x, y;
        __builtin_memcpy(&x, &a.w, 16); __builtin_memcpy(&y, &b.w, 16);
        return __builtin_amdgcn_mfma_f32_32x32x16_f16(x, y, c, 0, 0, 0);
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) c = __builtin_amdgcn_mfma_f32_32x32x2f32(a.w[j], b.w[j], c, 0, 0, 0);
        return c;
    }
}

__device__ __forceinline__ f32x16 zeros16() {
    f32x16 z;
#pragma unroll
    for (int i = 0; i < 16; ++i) z[i] = 0.0f;
    return z;
}

// Registers 8 x .. 8 x + 7 of an accumulator as a B operand: rounded to the storage type, nearest even
template <typename D> __device__ __forceinline__ Frag<D> to_frag(const f32x16& c, int x) {
    Frag<D> f;
    if constexpr (D::size == 4) {
#pragma unroll
        for (int j = 0; j < 8; ++j) f.w[j] = c[8 * x + j];
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const f32x2 p = {c[8 * x + 2 * j], c[8 * x + 2 * j + 1]};
            if constexpr (std::is_same<D, BF16>::value) { const bf16x2 r = __builtin_convertvector(p, bf16x2); uint32_t u; __builtin_memcpy(&u, &r, 4); f.w[j] = u; }
            else { const f16x2 r = __builtin_convertvector(p, f16x2); uint32_t u; __builtin_memcpy(&u, &r, 4); f.w[j] = u; }
        }
    }
    return f;
}

// The larger, and the sum, of a value of lane l and one of lane l ^ 32: the two lanes that share a column of C
__device__ __forceinline__ float halves_max(float x) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float halves_sum(float x) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// A tile in LDS: rows of DP elements (head_dim, filled up with zeros to a multiple of 32) in units of 16 bytes, four of them (64 bytes of a row) side by side, and
// the same four of four rows: slabs of 256 bytes.  Within the four the places are exchanged by the number of the row's four (xor), so that neither way of reading
// meets a bank twice: 16 lanes that read one unit of 16 rows (Reader::rows) hit 16 different groups of four banks, and so do the 32 lanes that read four
// consecutive units of four rows (Reader::columns).  All that a lane adds to its own address for other rows, steps or columns is then a constant of the
// instruction.  And the loads that fill it, whose lanes go through LDS in order, find 64 bytes of a row in every four lanes: with rows or pairs of units next to
// one another instead a load takes a cycle a lane (16 and 30 bytes a cycle and CU instead of 45).
template <typename D, int DP> struct Tile {
    static constexpr int kUnitElems = 16 / D::size;
    static constexpr int kUnits = DP / kUnitElems;
    static constexpr int kRowBytes = kUnits * 16;
    static_assert(kUnits % 4 == 0, "whole slabs");
    __device__ static __forceinline__ uint32_t place(uint32_t row, uint32_t unit) {
        return (row >> 2) * (kUnits * 64) + (unit >> 2) * 256u + (row & 3u) * 64u + ((unit ^ (row >> 2)) & 3u) * 16u;
    }
    // the other way round: which unit of which row is the p-th
    __device__ static __forceinline__ void at_place(uint32_t p, uint32_t& row, uint32_t& unit) {
        const uint32_t fours = (p >> 4) / (kUnits / 4);
        row = 4 * fours + ((p >> 2) & 3u);
        unit = 4 * ((p >> 4) % (kUnits / 4)) + ((p ^ fours) & 3u);
    }
};

// LDS by its bytes.  The kernels hand the buffer that is read and the one that is being filled to a step as __restrict pointers: that is how the compiler
// knows that a read need not wait for the loads on their way into the other.
typedef LSP_SHARED_AS uint8_t* Lds;
template <typename V> __device__ __forceinline__ V lds_read(Lds at) { return *(const LSP_SHARED_AS V*)at; }
template <typename V> __device__ __forceinline__ void lds_write(Lds at, V x) { *(LSP_SHARED_AS V*)at = x; }

// All loads into LDS that this wave has asked for have arrived, and every wave has said so.
__device__ __forceinline__ void arrived_for_all() {
    __builtin_amdgcn_s_waitcnt(0x0F70);                               // vmcnt(0)
    __syncthreads();
}

// Orders for the scheduler: so many matrix instructions, LDS reads, vector instructions next
template <int N> __device__ __forceinline__ void then_matrix() { __builtin_amdgcn_sched_group_barrier(0x008, N, 0); }
template <int N> __device__ __forceinline__ void then_reads() { __builtin_amdgcn_sched_group_barrier(0x100, N, 0); }
template <int N> __device__ __forceinline__ void then_vector() { __builtin_amdgcn_sched_group_barrier(0x402, N, 0); }

// Where a lane reads in a tile: computed once, the rest are constants.
template <typename D, int DP> struct Reader {
    using T = Tile<D, DP>;
    uint32_t row_at[2], column_at[2];
    __device__ __forceinline__ explicit Reader(int lane) {
        const uint32_t row = lane & 31, h = (uint32_t)lane >> 5;
#pragma unroll
        for (int x = 0; x < 2; ++x) {
            if constexpr (D::size == 2) {
                row_at[x] = T::place(row, 2 * x + h);                                     // even and odd steps
                const uint32_t unit = ((lane >> 4) & 1) * 2 + ((lane & 3) >> 1);
                column_at[x] = T::place(8 * x + 4 * h + ((lane >> 2) & 3), unit) + (lane & 1) * 8u;
            } else {
                row_at[x] = T::place(row, 2 * h + x);                                     // the two units of a step
                column_at[x] = T::place(8 * x + 4 * h, (lane & 31) >> 2) + (lane & 3) * 4u;
            }
        }
    }
    // A (or B) operand whose rows (columns) are rows ROW0 + 0..31 of the tile and whose k are its columns 16 ks + 0..15 (lane half h: 8 h + 0..7)
    __device__ __forceinline__ Frag<D> rows(Lds tile, int row0, int ks) const {
        Frag<D> f;
        const Lds t = tile + row0 / 4 * (T::kUnits * 64);
        if constexpr (D::size == 2) f.w = lds_read<u32x4>(t + row_at[ks & 1] + (ks >> 1) * 256);
        else {
            const f32x4 a = lds_read<f32x4>(t + row_at[0] + ks * 256), b = lds_read<f32x4>(t + row_at[1] + ks * 256);
#pragma unroll
            for (int j = 0; j < 4; ++j) { f.w[j] = a[j]; f.w[4 + j] = b[j]; }
        }
        return f;
    }
    // A operand whose rows are columns 32 ct + 0..31 of the tile and whose k are its rows ROW0 + 0..15, in the order that the accumulators have
    // them.  In 16 bits the transposing read does it: 16 lanes hold four rows of 16 columns, four columns each, and each gets one column of the four rows.
    __device__ __forceinline__ Frag<D> columns(Lds tile, int row0, int ct) const {
        Frag<D> f;
        const Lds t = tile + row0 / 4 * (T::kUnits * 64);
        if constexpr (D::size == 2) {
#pragma unroll
            for (int x = 0; x < 2; ++x) {
                const s16x4 v = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LSP_SHARED_AS s16x4*)(t + column_at[x] + ct * 256));
                u32x2 u;
                __builtin_memcpy(&u, &v, 8);
                f.w[2 * x] = u[0]; f.w[2 * x + 1] = u[1];
            }
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) f.w[j] = lds_read<float>(t + column_at[j >> 2] + ct * 512 + (j & 3) * 64);
        }
        return f;
    }
};

typedef __amdgpu_buffer_rsrc_t Buffer;
// A buffer of 2 GiB from p on; offsets from 2^31 on are out of it, and loads there give zeros
__device__ __forceinline__ Buffer buffer_from(const void* p) {
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(p), 0, 0x80000000u, 0x00027000);
}
template <typename D> __device__ __forceinline__ const uint8_t* at(const Strided& s, int64_t b, int64_t position, int64_t head) {
    return static_cast<const uint8_t*>(s.p) + (b * s.batch + position * s.position + head * s.head) * D::size;
}

constexpr uint32_t kNowhere = 0x80000000u;

// ROWS rows of a tile, asked for straight into LDS: a wave's load fills 1 KiB of LDS in the order of its lanes, so a lane asks for the unit that
// belongs at its place.  Rows from `left` on and columns from head_dim on lie out of the buffer: zeros, and not read.  They have arrived when vmcnt
// says so.
template <typename D, int DP, int ROWS, int NT> struct Fetch {
    using T = Tile<D, DP>;
    static constexpr int kWaves = NT / 64, kLoads = ROWS * T::kUnits / 64, kCount = (kLoads + kWaves - 1) / kWaves;
    static_assert(ROWS * T::kUnits % 64 == 0, "whole loads");
    uint32_t off[kCount];                                                                 // of this lane, from the tile's first row on
    int row[kCount];
    __device__ __forceinline__ void setup(uint32_t row_bytes, int head_dim, int wave, int lane) {
#pragma unroll
        for (int i = 0; i < kCount; ++i) {
            uint32_t r, unit;
            T::at_place((i * kWaves + wave) * 64 + lane, r, unit);
            row[i] = (int)r;
            off[i] = (int)unit * T::kUnitElems < head_dim ? r * row_bytes + unit * 16u : kNowhere;
        }
    }
    __device__ __forceinline__ void operator()(const void* first_row, int left, Lds tile, int wave) const {
        const Buffer b = buffer_from(first_row);
#pragma unroll
        for (int i = 0; i < kCount; ++i) {
            if (kLoads % kWaves && i * kWaves + wave >= kLoads) break;
            const uint32_t o = row[i] < left ? off[i] : kNowhere;
            __builtin_amdgcn_raw_ptr_buffer_load_lds(b, (LSP_SHARED_AS void*)(tile + (i * kWaves + wave) * 1024u), 16, (int)o, 0, 0, 0);
        }
    }
};

// fp32: operands straight from the lane's own row (a pointer to it, or NULL: zeros), columns 16 ks + 8 h + 0..7.  There the matrix instructions take so long that the
// way through LDS (below) only adds its latency: 37 instead of 41 us for the three passes of 8 heads of 64 x 64 x 64.
__device__ __forceinline__ Frag<F32> global_frag(const uint8_t* row, int ks, int head_dim, int lane) {
    const int col = 16 * ks + 8 * (lane >> 5);
    Frag<F32> f;
    if (row && col < head_dim) {
        const f32x4 a = *reinterpret_cast<const f32x4*>(row + col * 4), b = *reinterpret_cast<const f32x4*>(row + col * 4 + 16);
#pragma unroll
        for (int j = 0; j < 4; ++j) { f.w[j] = a[j]; f.w[4 + j] = b[j]; }
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) f.w[j] = 0.0f;
    }
    return f;
}

// The 32 rows of a wave on their way into 32 rows of LDS of its own, from where Reader::rows makes operands of them: a wave's loads find whole lines, where
// each lane asking for its own row would take a cycle a lane.  `offset(r)`: bytes from the buffer's begin to row r of the 32, or kNowhere for a row of zeros.
template <typename D, int DP, typename Offset> __device__ __forceinline__ void fetch_wave_rows(const Buffer& b, Lds at, int head_dim, int lane, Offset&& offset) {
    using T = Tile<D, DP>;
#pragma unroll
    for (int i = 0; i < T::kUnits / 2; ++i) {
        uint32_t r, unit;
        T::at_place(i * 64 + lane, r, unit);
        const uint32_t o = (int)unit * T::kUnitElems < head_dim ? offset(r) : kNowhere;
        __builtin_amdgcn_raw_ptr_buffer_load_lds(b, (LSP_SHARED_AS void*)(at + i * 1024u), 16, (int)(o + unit * 16u), 0, 0, 0);
    }
}

// And the way back: a wave's results, columns 8 (i / 4) + 4 h + i % 4 of 32 c + .. in registers i of v[c] and rows across lanes, as rows of the storage type: through
// 32 rows of LDS of its own, so that stores are of whole lines too.  `row(r)`: where row r of the 32 goes, or NULL.
template <typename D, int DP, typename Row> __device__ __forceinline__ void store_wave_rows(const f32x16 (&v)[DP / 32], float factor, Lds at, int head_dim, int lane, Row&& row) {
    using T = Tile<D, DP>;
    const uint32_t mine = lane & 31, h = (uint32_t)lane >> 5;
#pragma unroll
    for (int c = 0; c < DP / 32; ++c)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            const float x[4] = {v[c][4 * g] * factor, v[c][4 * g + 1] * factor, v[c][4 * g + 2] * factor, v[c][4 * g + 3] * factor};
            if constexpr (D::size == 4) lds_write<f32x4>(at + T::place(mine, 8 * c + 2 * g + h), f32x4{x[0], x[1], x[2], x[3]});
            else {
                u32x2 w;
                w[0] = (uint32_t)narrow<D>(x[0]) | (uint32_t)narrow<D>(x[1]) << 16;
                w[1] = (uint32_t)narrow<D>(x[2]) | (uint32_t)narrow<D>(x[3]) << 16;
                lds_write<u32x2>(at + T::place(mine, 4 * c + g) + h * 8u, w);
            }
        }
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
#pragma unroll
    for (int i = 0; i < T::kUnits / 2; ++i) {
        uint32_t r, unit;
        T::at_place(i * 64 + lane, r, unit);
        const u32x4 w = lds_read<u32x4>(at + (i * 64 + lane) * 16);
        uint8_t* p = row(r);
        if (p && (int)unit * T::kUnitElems < head_dim) *reinterpret_cast<u32x4*>(p + unit * 16u) = w;
    }
}

// Four consecutive elements of an output row
template <typename D> __device__ __forceinline__ void store_four(uint8_t* p, float a, float b, float c, float d) {
    typename D::elem t[4] = {narrow<D>(a), narrow<D>(b), narrow<D>(c), narrow<D>(d)};
    if constexpr (D::size == 2) { u32x2 w; __builtin_memcpy(&w, t, 8); *reinterpret_cast<u32x2*>(p) = w; }
    else { u32x4 w; __builtin_memcpy(&w, t, 16); *reinterpret_cast<u32x4*>(p) = w; }
}

__device__ __forceinline__ int valid_length(const int32_t* lens, int b, int most) { return lens ? min(max(lens[b], 0), most) : most; }

// What workgroup `block` does: a tile of a unit (a head, or a part of one).  Workgroups go round the eight XCDs, each with an L2 of its own: an XCD gets whole units, so
// that the workgroups that read the same rows share an L2, and goes through them tile by tile: tile 0 of all its units first, the one with the most work.
__device__ __forceinline__ void work_of_block(uint32_t block, uint32_t units, uint32_t tiles, int& unit, int& tile) {
    const uint32_t xcd = block & 7u, nth = block >> 3;
    if (units % 8u == 0) {
        const uint32_t share = units / 8u;
        tile = (int)(nth / share);
        unit = (int)(xcd * share + nth % share);
    } else {                                                                              // runs of (unit, tile)
        const uint32_t items = units * tiles, share = items >> 3, rest = items & 7u, item = xcd * share + min(xcd, rest) + nth;
        unit = (int)(item / tiles);
        tile = (int)(item % tiles);
    }
}
#endif

}  // namespace lsp

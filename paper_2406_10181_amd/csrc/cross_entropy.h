// Arguments of the cross-entropy kernels.  Those with products in them are in cross_entropy_products.h, the others in cross_entropy.hip.
//
// A block of rows goes through five kernels.  k_loss_pack copies the rows of H that count, one behind the other, so that rows that do not count cost nothing and are not
// read.  k_loss_logits multiplies W by them; z[v][row] is in registers with the row across lanes and a piece of the vocabulary (a wave's part of the tile)
// in the lane's registers, so that a piece's maximum and sum of exponentials take no LDS.  The exponentials, relative to the piece's maximum, are stored in 16 bits (fp32: in 32): whatever
// the size of z they keep its digits, where z itself in 16 bits would be off by a hundredth of a unit and p by a percent.  k_loss_rows makes the rows' maxima, sums and losses of
// the pieces (k_loss_dz, where they are few), maximum and sum apart: nothing that p is made of is rounded at the size of z; k_loss_dz turns the exponentials into the gradient of z in place; k_loss_back multiplies that by W and by H.
//
// Of the roundings on the way one would be seen in 16 bits, that of a target's dz, which is most of its row: dH gets what it takes off, times the target's row of W, behind the products; for
// dW the gradient's scale keeps it small, and of up to 32 rows what is taken off has rows of its own.  dH is as far from the exact one as a result that is rounded once, dW up to 1.4 times as
// far.  Weights of fp16 that differ by 2^18 and more cost the small ones' rows digits: one scale serves all, since dW's products run over the rows.
//
// 6 rows width vocab operations in all: keeping 16 bits an exponential, 2 bytes written, read, written and read twice, costs less than a second product
// would.  4096 rows, width 4096, 32000 words in bf16: logits 0.79-0.85 ms, dz 0.08 (6.5 TB/s), both gradients 1.55-1.65 ms, 2.44 ms in all, 1320 TFLOP/s, which is what the power allows of
// products of random numbers: large plain products reach 1320 to 1580 with W's or H's rows along k, and 1100 to 1390 where an operand lies across.
// The blocks are as large as kLossBytes allows, and where there are several, dW is added up in fp32.
#pragma once

#include "attention.h"
#include "rows.h"

namespace lsp {

constexpr size_t kLossBytes = (size_t)1 << 30;    // of exponentials, at most (but for one tile of rows)

struct LossArgs {
    const void *H, *W;
    const int64_t* targets;
    const float* weights;
    float *losses, *logs;
    void *dH, *dW;
    int64_t h_stride, w_stride, dh_stride, dw_stride;
    int64_t rows;
    int32_t width, vocab;
    float smoothing, z_loss, scale;
    // workspace
    int32_t* count;              // [4]: rows that count; bits of the largest gradient of z that there can be (fp16), and of the largest weight; one of padding
    int32_t* index;              // [rows]: which they are
    uint8_t* packed;             // [block_rows][width] of the storage type: the block's rows
    int32_t* target;             // [block_rows]
    float *top, *sum, *plain;    // [pieces][block_rows]: a piece's maximum, sum of exponentials, sum of z (with smoothing only)
    float *hit;                  // [block_rows]: z[target]
    float *row_top, *row_sum;    // [block_rows]: a row's maximum t and the sum of exp(z - t)
    float *factor;               // [block_rows]: scale * weight
    float *left;                 // [block_rows], 16 bits: what the rounding of dz[row][target] took off
    uint8_t* e;                  // [block_rows][padded]
    float* dh_parts;             // [dh_splits][block_rows][width], where there are several; or more of fewer rows: parts_of_dh()
    float* dw_sum;               // [vocab][width], where there are several blocks of rows and dW is not fp32
    // plan
    int32_t block_rows, padded;  // multiples of 256
    int32_t blocks, block;       // blocks of rows, and which this is
    int32_t pieces, piece;       // pieces of the vocabulary, of so many
    int32_t tile[2];             // 256 (16 bits only), 128, 64 or 32: of the logits, and of dH and dW
    int32_t dh_splits, dh_room;  // parts of the vocabulary that dH is made of; tiles of rows times parts
    int32_t dw_first;            // whether dW's workgroups come before dH's, and how many of the one come before the other
    int32_t first_blocks;
    int32_t train, twice;        // twice: each row has a second one behind the last, with that alone
};

void plan_loss(LossArgs& a, lsp_dtype dtype);
size_t loss_workspace(LossArgs& a, lsp_dtype dtype, uint8_t* base);     // the bytes; places the pieces where base is not NULL
hipError_t launch_loss(LossArgs& a, lsp_dtype dtype, hipStream_t st);

template <typename D> hipError_t launch_loss_logits(const LossArgs& a, hipStream_t st);
template <typename D> hipError_t launch_loss_back(const LossArgs& a, hipStream_t st);

#if defined(__HIPCC__)
constexpr float kLossLog2e = 1.44269504088896341f;
// What an exponential is stored in: fp16 for bf16 too, whose digits would be three fewer.  It counts as 2^15 at the top, so that what is 2^-29 of the largest still has all its digits.
template <typename D> using LossExp = std::conditional_t<std::is_same<D, F32>::value, F32, F16>;
template <typename D> constexpr float kLossTop = std::is_same<D, F32>::value ? 1.0f : 32768.0f;
template <typename D> constexpr float kLossTopLog2 = std::is_same<D, F32>::value ? 0.0f : 15.0f;

// Rows of this block that count
__device__ __forceinline__ int rows_of_block(const LossArgs& a) {
    return min(max(*as_const<int32_t>(a.count) - a.block * a.block_rows, 0), a.block_rows);
}
// How many rows dW is a product of
__device__ __forceinline__ int rows_of_dw(const LossArgs& a, int rows) { return a.twice ? 2 * rows : rows; }
// Parts of the vocabulary that dH is made of, and the rows between two parts' sums: where fewer rows count than there are, their tiles get the workgroups (and the room) that the others would
// have had.  (3001 rows of which 1800 count, width 1000, 50021 words, fp16: dH in a launch of its own 183 us, with the parts planned for all rows 230.)
struct LossParts { int splits, rows; };
__device__ __forceinline__ LossParts parts_of_dh(const LossArgs& a, int rows) {
    const int tile = a.tile[1], tiles = (rows + tile - 1) / tile;
    return {a.dh_splits > 1 && tiles > 0 ? a.dh_room / tiles : 1, tiles * tile};
}
// What the gradient of z is multiplied by in 16 bits; the products of it are divided by that.  Its mantissa brings the gradient of a target of the largest weight to just below a power of two, where rounding is off
// by the least (of equal weights by 2^-9 at most in bf16, otherwise by up to 2^-8).  (It is 1 at most: no gradient grows out of range by it.)  fp16: and its power of two brings the largest
// that there can be below 2^14.
template <typename D> __device__ __forceinline__ float gradient_scale(const LossArgs& a) {
    if constexpr (D::size == 4) return 1.0f;
    const uint32_t usual = __float_as_uint(fabsf(a.scale * as_const<float>(a.count)[2] * (1.0f - a.smoothing)));
    const float mantissa = usual < 0x00800000u || usual >= 0x7F800000u ? 1.0f : __uint_as_float((usual & 0x7FFFFFu) | 0x3F800000u), scale = 0.99609375f / mantissa;
    if constexpr (std::is_same<D, BF16>::value) return scale;
    const uint32_t largest = as_const<uint32_t>(a.count)[1];                              // an fp32 number's bits
    const int exponent = max((int)(largest >> 23) - 127, -100);
    return largest == 0 || largest >= 0x7F800000u ? scale : scale * __uint_as_float((uint32_t)(127 + 13 - exponent) << 23);
}

// Four elements of 16 bits
template <typename D> __device__ __forceinline__ f32x4 four_of(const uint8_t* at) {
    const u32x2 w = *reinterpret_cast<const u32x2*>(at);
    Packed<D> p;
    p.w[0] = w[0]; p.w[1] = w[1]; p.w[2] = p.w[3] = 0;
    const Eight x = widen_eight<D>(p);
    return f32x4{x.x[0], x.x[1], x.x[2], x.x[3]};
}
#endif

}  // namespace lsp

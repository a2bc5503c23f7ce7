// y := drop(x), the mask made on the way from (seed, offset, place) and never stored; the backward pass is the same call on the
// gradient.
//
// A thread takes eight elements that follow one another in a row: one call of the generator, one load and one store of 16 (or, in
// fp32, 32) bytes.  Rows need not be a multiple of anything: each begins a new block of eight, so that the mask of a row does not
// depend on how the others lie; where rows begin off the 16-byte steps the loads are unaligned ones, and the last block of a row
// goes in pieces of four, two and one.
//
// Bound by memory: 4096 x 11008 bf16, 180 MB, 30 us, 6.0 TB/s (the generator's 28 products of 32 bits for eight elements hide behind it).
#include "philox.h"
#include "rows.h"

namespace lsp {

constexpr int kDropThreads = 256;

template <typename D>
__global__ __launch_bounds__(kDropThreads) void k_dropout(const typename D::elem* x, typename D::elem* y, int64_t rows, int32_t width, uint32_t blocks,
                                                          Dropout drop) {
    const uint64_t n = (uint64_t)blockIdx.x * kDropThreads + threadIdx.x;          // number of the block of eight
    if (n >= (uint64_t)rows * blocks) return;
    const uint64_t row = n / blocks;
    const int col = (int)(n - row * blocks) * 8;
    const int left = width - col;
    const typename D::elem* from = x + row * (uint64_t)width + col;
    Eight v = load_eight<D>(from, left);
    const u32x4 w = philox((uint32_t)n, (uint32_t)(n >> 32), 0, drop.offset, drop.key0, drop.key1);
#pragma unroll
    for (int e = 0; e < 8; ++e) v.x[e] = philox_word(w, e) < drop.limit ? 0.0f : v.x[e] * drop.scale;
    store_eight<D>(y + row * (uint64_t)width + col, v, left);
}

hipError_t launch_dropout(const void* x, void* y, int64_t rows, int64_t width, const Dropout& drop, lsp_dtype dtype, hipStream_t st) {
    const uint64_t blocks = (uint64_t)(width + 7) / 8, total = blocks * (uint64_t)rows;
    const dim3 grid((unsigned)((total + kDropThreads - 1) / kDropThreads));
    if (dtype == LSP_F32) hipLaunchKernelGGL(k_dropout<F32>, grid, dim3(kDropThreads), 0, st, static_cast<const float*>(x), static_cast<float*>(y), rows, (int32_t)width, (uint32_t)blocks, drop);
    else if (dtype == LSP_F16) hipLaunchKernelGGL(k_dropout<F16>, grid, dim3(kDropThreads), 0, st, static_cast<const uint16_t*>(x), static_cast<uint16_t*>(y), rows, (int32_t)width, (uint32_t)blocks, drop);
    else hipLaunchKernelGGL(k_dropout<BF16>, grid, dim3(kDropThreads), 0, st, static_cast<const uint16_t*>(x), static_cast<uint16_t*>(y), rows, (int32_t)width, (uint32_t)blocks, drop);
    return hipGetLastError();
}

}  // namespace lsp

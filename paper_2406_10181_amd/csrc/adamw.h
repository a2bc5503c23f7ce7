// Arguments of the optimizer step's kernel (adamw.hip).
#pragma once

#include "lsp_internal.h"

namespace lsp {

constexpr int kAdamwThreads = 256, kAdamwElements = 8 * kAdamwThreads;   // of a workgroup
constexpr int kAdamwBlock = 256;                                        // elements that share a scale
constexpr int kMaxItems = 32;                                           // tensors of a launch: what fits into its arguments

struct AdamwStep { float one_minus_beta1, beta1, one_minus_beta2, beta2, inv_c1, inv_c2, eps, rate; };

struct AdamwGroup {
    AdamwStep      step;
    const float*   grad_scale;
    int64_t        pad;
    double         one_minus_beta1, beta1, one_minus_beta2, beta2;      // states in 8 bits
    uint32_t       first[kMaxItems];               // workgroup that each tensor begins with; past the last tensor UINT32_MAX
    lsp_adamw_item item[kMaxItems];
};
static_assert(sizeof(AdamwGroup) <= 4096, "a launch's arguments");

hipError_t launch_adamw(const AdamwGroup& g, uint32_t blocks, bool bits8, hipStream_t st);

}  // namespace lsp

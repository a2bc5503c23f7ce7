// Arguments of the optimizer step's kernel (adamw.hip).
#pragma once

#include "lsp_internal.h"

namespace lsp {

constexpr int kAdamwThreads = 256, kAdamwRounds = 2, kAdamwElements = 8 * kAdamwThreads * kAdamwRounds;   // of a workgroup
constexpr int kAdamwBlock = 256;                                        // elements that share a scale
constexpr int kMaxItems = 32;                                           // tensors of a launch: what fits into its arguments

// With c1 = 1 - beta1^step and c2 alike:  rate (m / c1) / (sqrt(v / c2) + eps) = (rate sqrt(c2) / c1) m / (sqrt(v) + eps sqrt(c2))
struct AdamwStep { float one_minus_beta1, beta1, one_minus_beta2, beta2, eps, rate, decay_rate, pad; };

struct AdamwGroup {
    AdamwStep      step;
    const float*   grad_scale;
    int64_t        pad;
    double         one_minus_beta1, beta1, one_minus_beta2, beta2;      // states in 8 bits
    int32_t        first[kMaxItems];               // workgroup that each tensor begins with; past the last tensor INT32_MAX
    lsp_adamw_item item[kMaxItems];
};
static_assert(sizeof(AdamwGroup) <= 4096, "a launch's arguments");

hipError_t launch_adamw(const AdamwGroup& g, uint32_t blocks, bool bits8, hipStream_t st);

}  // namespace lsp

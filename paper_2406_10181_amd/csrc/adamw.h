// Arguments of the optimizer step's kernel (adamw.hip).
#pragma once

#include <type_traits>

#include "lsp_internal.h"

namespace lsp {

constexpr int kAdamwThreads = 256, kAdamwRounds = 2, kAdamwElements = 8 * kAdamwThreads * kAdamwRounds;   // of a workgroup
constexpr int kAdamwBlock = 256;                                        // elements that share a scale

// With c1 = 1 - beta1^step and c2 alike:  rate (m / c1) / (sqrt(v / c2) + eps) = (rate sqrt(c2) / c1) m / (sqrt(v) + eps sqrt(c2))
struct AdamwStep { float one_minus_beta1, beta1, one_minus_beta2, beta2, eps, rate, decay_rate; };

// A launch's arguments, as many tensors as fit into them.  (200 tensors of 4096 elements: 14 us, with 32 of them a launch 32.)
struct AdamwTensor {
    void*       param;
    const void* grad;
    void*       m;
    void*       v;
    float*      master;
    int64_t     elements;
    float       rate_factor, decay;
};
struct AdamwTensor8 : AdamwTensor { float *m_scale, *v_scale; };
constexpr int64_t kAdamwSizes = (int64_t)1 << 40;                       // elements below this, dtype and grad_dtype above
template <bool BITS8> struct AdamwGroup {
    static constexpr int kItems = BITS8 ? 52 : 64;
    AdamwStep    step;
    const float* grad_scale;
    double       one_minus_beta1, beta1, one_minus_beta2, beta2;        // states in 8 bits
    int32_t      first[kItems];                                         // workgroup that each tensor begins with; past the last tensor INT32_MAX
    std::conditional_t<BITS8, AdamwTensor8, AdamwTensor> item[kItems];
};
static_assert(sizeof(AdamwGroup<false>) <= 4096 && sizeof(AdamwGroup<true>) <= 4096, "a launch's arguments");

template <bool BITS8> hipError_t launch_adamw(const AdamwGroup<BITS8>& g, uint32_t blocks, hipStream_t st);

}  // namespace lsp

// Arguments of the rotary kernels (rotary.hip).
#pragma once

#include "attention.h"

namespace lsp {

constexpr int kRotaryTokens = 16;                   // most tokens of a workgroup
// What is done head by head alike: queries, keys, and (forward) values, which are only moved
struct RotarySegment {
    Strided x, y;                                   // forward: from and to; backward: what was normed, and the gradient that arrives
    Strided out;                                    // backward: the gradient that is made
    const void *weight, *bias;
    float *weight_sum, *bias_sum;                   // backward: gradients of these, or NULL
    int32_t heads, placed;                          // placed: y has places of a cache, not positions of the text
    int32_t tokens, parts;                          // of a workgroup; workgroups that share the tokens' heads
    int32_t first, blocks;                          // its workgroups
};
struct RotaryArgs {
    RotarySegment segment[3];
    const float* frequencies;
    const int32_t *positions, *starts, *lens;
    float* partial;                                 // backward: [workgroups][2][head_dim], sums for weight and bias
    int32_t batch, length, cache, head_dim, rotated, neighbours, norm;
    int32_t segments, blocks;
    int32_t sums;                                   // backward: whether any gradient of a weight or bias is asked for
    float eps;
};

void plan_rotary(RotaryArgs& a, bool backward);
size_t rotary_partial_bytes(const RotaryArgs& a);
hipError_t launch_rotary(const RotaryArgs& a, bool backward, lsp_dtype dtype, hipStream_t st);

}  // namespace lsp

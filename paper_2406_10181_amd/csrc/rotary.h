// Arguments of the rotary kernels (rotary.hip).
#pragma once

#include "attention.h"

namespace lsp {

struct RotaryArgs {
    Strided q, k, v, qr, kr, vr;                    // backward: qr, kr are dQr, dKr and v, vr are dQ, dK
    const void *q_w, *k_w, *q_b, *k_b;
    const float* frequencies;
    const int32_t *positions, *starts, *lens;
    float* partial;                                 // backward: [workgroups][4][head_dim], sums of q_weight, k_weight, q_bias, k_bias
    float* grads[4];                                // NULL: not asked for
    int32_t batch, length, cache, heads, kv_heads, head_dim, rotated, neighbours, norm;
    int32_t rows;                                   // of a token: heads of Q, of K and (forward, if there is a V) of V
    int32_t parts;                                  // lane groups that share a token's rows
    int32_t sums;                                   // backward: whether any of grads is asked for
    int32_t blocks;                                 // backward: workgroups, each with a part of the sums
    float eps;
};

void plan_rotary(RotaryArgs& a, bool backward);
size_t rotary_partial_bytes(const RotaryArgs& a);
hipError_t launch_rotary(const RotaryArgs& a, bool backward, lsp_dtype dtype, hipStream_t st);

}  // namespace lsp

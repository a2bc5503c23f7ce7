// Argument checks that the operators of a training step share (host only).
#pragma once

#include <algorithm>
#include <cmath>

#include "attention.h"

namespace {

inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
inline bool known(lsp_dtype t) { return t == LSP_F32 || t == LSP_F16 || t == LSP_BF16; }
inline int elem_size(lsp_dtype t) { return t == LSP_F32 ? 4 : 2; }
inline bool rate(float p) { return p >= 0.0f && p < 1.0f; }                       // (false for a NaN)
inline int done(hipError_t e) { return e == hipSuccess ? LSP_OK : lsp::note_hip_error(e); }

// Whether every row has a place of its own: each axis steps over all that the axes of smaller strides span
inline bool rows_apart(const int64_t (&s)[3], const int64_t (&count)[3], int64_t dim) {
    int order[3] = {0, 1, 2};
    std::sort(order, order + 3, [&](int i, int j) { return s[i] < s[j]; });
    __int128 span = dim;
    for (const int k : order) {
        if (count[k] == 1) continue;                                      // (not used)
        if (s[k] < span) return false;
        span += (__int128)s[k] * (count[k] - 1);
    }
    return true;
}

// One operand's strides: multiples of 16 bytes, positions less than 8 MiB apart (a tile is addressed with 32 bits), batches and heads anywhere
// below 2^40 elements; what is written has a place of its own for every row.
inline int check_strides(const int64_t (&s)[3], int64_t batch, int64_t positions, int64_t heads, int32_t dim, lsp_dtype t, bool written) {
    const int64_t per = 16 / elem_size(t);
    const int64_t count[3] = {batch, positions, heads};
    for (int k = 0; k < 3; ++k) {
        if (count[k] == 1) continue;                                      // (not used)
        if (s[k] < 0 || s[k] > ((int64_t)1 << 40)) return LSP_ERR_SHAPE;
        if (s[k] % per) return LSP_ERR_ALIGN;
    }
    if (positions > 1 && s[1] * elem_size(t) >= (8 << 20)) return LSP_ERR_SHAPE;
    if (written && !rows_apart(s, count, dim)) return LSP_ERR_SHAPE;
    return LSP_OK;
}

inline lsp::Strided strided(const void* p, const int64_t (&s)[3], int64_t batch, int64_t positions, int64_t heads) {
    return {p, batch > 1 ? s[0] : 0, positions > 1 ? s[1] : 0, heads > 1 ? s[2] : 0};
}

inline bool norm_kind(int32_t k) { return k == LSP_NORM_NONE || k == LSP_NORM_RMS || k == LSP_NORM_LAYER; }

// Whether an output over an input lies on it row by row
inline bool on_it(const void* in, int64_t in_stride, const void* out, int64_t out_stride, int64_t rows) { return in != out || rows == 1 || in_stride == out_stride; }

}  // namespace

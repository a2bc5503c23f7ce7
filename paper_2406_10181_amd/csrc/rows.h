// Eight consecutive elements of a row, widened to fp32: the unit in which the row-wise kernels (dropout, residual norm) work.
// A row may begin at any element, so the addresses are aligned to one element only; the loads and stores are wide all the same.
#pragma once

#include "lsp_internal.h"

#if defined(__HIPCC__)
namespace lsp {

struct Eight { float x[8]; };

// (as vectors of words: the compiler keeps them whole)
typedef u32x4 u32x4_any2 __attribute__((aligned(2)));
typedef u32x4 u32x4_any4 __attribute__((aligned(4)));

template <typename D> __device__ __forceinline__ Eight load_eight(const typename D::elem* p, int left) {
    Eight r;
    if (left >= 8) {
        typename D::elem t[8];
        if constexpr (D::size == 2) {
            const u32x4 w = *reinterpret_cast<const u32x4_any2*>(p);
            __builtin_memcpy(t, &w, 16);
        } else {
            const u32x4 a = *reinterpret_cast<const u32x4_any4*>(p), b = *reinterpret_cast<const u32x4_any4*>(p + 4);
            __builtin_memcpy(t, &a, 16); __builtin_memcpy(t + 4, &b, 16);
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) r.x[e] = widen<D>(t[e]);
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) r.x[e] = e < left ? widen<D>(p[e]) : 0.0f;
    }
    return r;
}

template <typename D> __device__ __forceinline__ void store_eight(typename D::elem* p, const Eight& r, int left) {
    typename D::elem t[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) t[e] = narrow<D>(r.x[e]);
    if (left >= 8) {
        if constexpr (D::size == 2) {
            u32x4 w;
            __builtin_memcpy(&w, t, 16);
            *reinterpret_cast<u32x4_any2*>(p) = w;
        } else {
            u32x4 a, b;
            __builtin_memcpy(&a, t, 16); __builtin_memcpy(&b, t + 4, 16);
            *reinterpret_cast<u32x4_any4*>(p) = a; *reinterpret_cast<u32x4_any4*>(p + 4) = b;
        }
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) if (e < left) p[e] = t[e];
    }
}

}  // namespace lsp
#endif

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
typedef u32x2 u32x2_any2 __attribute__((aligned(2)));
typedef u32x2 u32x2_any4 __attribute__((aligned(4)));
typedef uint32_t u32_any2 __attribute__((aligned(2)));

// The same as it lies in memory, in words (16-bit elements in arrays of their own would have a register each)
template <typename D> struct Packed { uint32_t w[2 * D::size]; };
template <typename D> __device__ __forceinline__ Packed<D> load_whole(const typename D::elem* p) {
    Packed<D> r;
    if constexpr (D::size == 2) {
        const u32x4 w = *reinterpret_cast<const u32x4_any2*>(p);
        __builtin_memcpy(r.w, &w, 16);
    } else {
        const u32x4 a = *reinterpret_cast<const u32x4_any4*>(p), b = *reinterpret_cast<const u32x4_any4*>(p + 4);
        __builtin_memcpy(r.w, &a, 16); __builtin_memcpy(r.w + 4, &b, 16);
    }
    return r;
}
// The last block of a row, of fewer than eight elements (or none): four, two and one of them, as the bits of `left` say
template <typename D> __device__ __forceinline__ Packed<D> load_part(const typename D::elem* p, int left) {
    const int n = max(left, 0);
    const bool four = n & 4, two = n & 2, one = n & 1;
    Packed<D> r;
    if constexpr (D::size == 2) {
        u32x2 a = {0, 0};
        uint32_t b = 0, c = 0;
        if (four) a = *reinterpret_cast<const u32x2_any2*>(p);
        if (two) b = *reinterpret_cast<const u32_any2*>(p + (n & 4));
        if (one) c = p[n & 6];
        r.w[0] = four ? a[0] : two ? b : c;
        r.w[1] = four ? a[1] : two ? c : 0u;
        r.w[2] = four ? (two ? b : c) : 0u;
        r.w[3] = four && two ? c : 0u;
    } else {
        u32x4 a = {0, 0, 0, 0};
        u32x2 b = {0, 0};
        uint32_t c = 0;
        if (four) a = *reinterpret_cast<const u32x4_any4*>(p);
        if (two) b = *reinterpret_cast<const u32x2_any4*>(p + (n & 4));
        if (one) c = __float_as_uint(p[n & 6]);
        r.w[0] = four ? a[0] : two ? b[0] : c;
        r.w[1] = four ? a[1] : two ? b[1] : 0u;
        r.w[2] = four ? a[2] : two ? c : 0u;
        r.w[3] = four ? a[3] : 0u;
        r.w[4] = four ? (two ? b[0] : c) : 0u;
        r.w[5] = four && two ? b[1] : 0u;
        r.w[6] = four && two ? c : 0u;
        r.w[7] = 0u;
    }
    return r;
}
template <typename D> __device__ __forceinline__ Packed<D> load_packed(const typename D::elem* p, int left) { return left >= 8 ? load_whole<D>(p) : load_part<D>(p, left); }
template <typename D> __device__ __forceinline__ float element(const Packed<D>& p, int e) {
    if constexpr (D::size == 4) return __uint_as_float(p.w[e]);
    else if constexpr (std::is_same<D, BF16>::value) return __uint_as_float(e & 1 ? p.w[e >> 1] & 0xFFFF0000u : p.w[e >> 1] << 16);
    else return widen<D>((uint16_t)(e & 1 ? p.w[e >> 1] >> 16 : p.w[e >> 1]));
}
template <typename D> __device__ __forceinline__ Eight widen_eight(const Packed<D>& p) {
    Eight r;
#pragma unroll
    for (int e = 0; e < 8; ++e) r.x[e] = element<D>(p, e);
    return r;
}
template <typename D> __device__ __forceinline__ Eight load_eight(const typename D::elem* p, int left) {
    return widen_eight<D>(load_packed<D>(p, left));
}

// Eight elements at p of which the first `first` belong to somebody else.  They are read with the others where that may be (`whole`, the same for all), so that nothing is
// put together from parts before it is needed, and otherwise are zeros; first = 8: zeros.
template <typename D> __device__ __forceinline__ Packed<D> load_ending(const typename D::elem* p, int first, bool whole) {
    Packed<D> r;
#pragma unroll
    for (int k = 0; k < 2 * D::size; ++k) r.w[k] = 0;
    if (first == 0 || (whole && first < 8)) r = load_whole<D>(p);
    else if (!whole) {
#pragma unroll
        for (int e = 1; e < 8; ++e) {
            if (e < first) continue;
            if constexpr (D::size == 4) r.w[e] = __float_as_uint(p[e]);
            else r.w[e >> 1] |= (uint32_t)p[e] << (16 * (e & 1));
        }
    }
    return r;
}

// Sum over a wave, in every lane.  Sums of 16 lanes and then of the four sixteens by moves between lanes that need no LDS.
template <int CTRL, int ROWS> __device__ __forceinline__ float plus_lane(float x) {
    return x + __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), CTRL, ROWS, 0xF, false));
}
__device__ __forceinline__ float wave_sum(float x) {
    x = plus_lane<0x111, 0xF>(x); x = plus_lane<0x112, 0xF>(x); x = plus_lane<0x114, 0xF>(x); x = plus_lane<0x118, 0xF>(x);   // row_shr 1, 2, 4, 8
    x = plus_lane<0x142, 0xA>(x); x = plus_lane<0x143, 0xC>(x);                                                               // row_bcast 15, 31
    return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(x), 63));
}

template <typename D> __device__ __forceinline__ Packed<D> narrow_eight(const Eight& r) {
    Packed<D> o;
    if constexpr (D::size == 4) {
#pragma unroll
        for (int e = 0; e < 8; ++e) o.w[e] = __float_as_uint(r.x[e]);
    } else {
#pragma unroll
        for (int k = 0; k < 4; ++k) o.w[k] = (uint32_t)narrow<D>(r.x[2 * k]) | (uint32_t)narrow<D>(r.x[2 * k + 1]) << 16;
    }
    return o;
}
template <typename D> __device__ __forceinline__ void store_whole(typename D::elem* p, const Packed<D>& o) {
    if constexpr (D::size == 2) {
        *reinterpret_cast<u32x4_any2*>(p) = u32x4{o.w[0], o.w[1], o.w[2], o.w[3]};
    } else {
        *reinterpret_cast<u32x4_any4*>(p) = u32x4{o.w[0], o.w[1], o.w[2], o.w[3]};
        *reinterpret_cast<u32x4_any4*>(p + 4) = u32x4{o.w[4], o.w[5], o.w[6], o.w[7]};
    }
}
// Eight elements but the first `first`
template <typename D> __device__ __forceinline__ void store_ending(typename D::elem* p, const Eight& r, int first) {
    const Packed<D> o = narrow_eight<D>(r);
    if (first == 0) { store_whole<D>(p, o); return; }
#pragma unroll
    for (int e = 1; e < 8; ++e) {
        if (e < first) continue;
        if constexpr (D::size == 4) p[e] = __uint_as_float(o.w[e]);
        else p[e] = (uint16_t)(o.w[e >> 1] >> (16 * (e & 1)));
    }
}
template <typename D> __device__ __forceinline__ void store_eight(typename D::elem* p, const Eight& r, int left) {
    const Packed<D> o = narrow_eight<D>(r);
    if (left >= 8) { store_whole<D>(p, o); return; }
    const int n = max(left, 0);
    const bool four = n & 4, two = n & 2;
    if constexpr (D::size == 2) {
        if (four) *reinterpret_cast<u32x2_any2*>(p) = u32x2{o.w[0], o.w[1]};
        if (two) *reinterpret_cast<u32_any2*>(p + (n & 4)) = four ? o.w[2] : o.w[0];
        if (n & 1) p[n & 6] = (uint16_t)(four ? (two ? o.w[3] : o.w[2]) : two ? o.w[1] : o.w[0]);
    } else {
        if (four) *reinterpret_cast<u32x4_any4*>(p) = u32x4{o.w[0], o.w[1], o.w[2], o.w[3]};
        if (two) *reinterpret_cast<u32x2_any4*>(p + (n & 4)) = four ? u32x2{o.w[4], o.w[5]} : u32x2{o.w[0], o.w[1]};
        if (n & 1) p[n & 6] = __uint_as_float(four ? (two ? o.w[6] : o.w[4]) : two ? o.w[2] : o.w[0]);
    }
}

}  // namespace lsp
#endif

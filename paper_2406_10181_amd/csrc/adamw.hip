// One step of AdamW over many tensors in a launch, states in fp32 or in 8 bits.
//
// Bound by memory: a bf16 element takes 22 bytes with states in fp32 (30 with an fp32 master) and 10 with states in 8 bits; nothing is read twice.  A thread
// takes eight elements that follow one another, so that every stream goes in loads of 8 to 32 bytes a lane, and 32 lanes have the 256 elements of a scale:
// its maximum goes through the 32 lanes without LDS.  A workgroup has 2048 elements of one tensor; the tensors' descriptors come with the launch (kMaxItems of
// them), so that a model's many small tensors take few launches and no memory of their own.
#include "adamw.h"
#include "rows.h"

namespace lsp {

// The largest of 32 lanes, in all of them.  (row_ror by 8, 4, 2, 1 in the sixteens, then the two halves of 32.)  fmaxf passes over a NaN.
template <int CTRL> __device__ __forceinline__ float max_lane(float x) {
    return fmaxf(x, __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), CTRL, 0xF, 0xF, false)));
}
__device__ __forceinline__ float max_of_32(float x) {
    x = max_lane<0x128>(x); x = max_lane<0x124>(x); x = max_lane<0x122>(x); x = max_lane<0x121>(x);
    return fmaxf(x, __int_as_float(__builtin_amdgcn_ds_swizzle(__float_as_int(x), 0x401F)));              // lane ^ 16
}

__device__ __forceinline__ Eight load_any(const void* p, int64_t at, int left, int dtype) {
    if (dtype == LSP_F32) return load_eight<F32>(static_cast<const float*>(p) + at, left);
    const uint16_t* q = static_cast<const uint16_t*>(p) + at;
    return dtype == LSP_F16 ? load_eight<F16>(q, left) : load_eight<BF16>(q, left);
}
__device__ __forceinline__ void store_any(void* p, int64_t at, const Eight& x, int left, int dtype) {
    if (dtype == LSP_F32) { store_eight<F32>(static_cast<float*>(p) + at, x, left); return; }
    uint16_t* q = static_cast<uint16_t*>(p) + at;
    if (dtype == LSP_F16) store_eight<F16>(q, x, left);
    else store_eight<BF16>(q, x, left);
}

// Eight bytes, of which `left` there are
__device__ __forceinline__ u32x2 load_codes(const uint8_t* p, int left) {
    if (left >= 8) return *reinterpret_cast<const u32x2*>(p);
    u32x2 w = {0, 0};
    for (int e = 0; e < left; ++e) w[e >> 2] |= (uint32_t)p[e] << (8 * (e & 3));
    return w;
}
__device__ __forceinline__ void store_codes(uint8_t* p, u32x2 w, int left) {
    if (left >= 8) { *reinterpret_cast<u32x2*>(p) = w; return; }
    for (int e = 0; e < left; ++e) p[e] = (uint8_t)(w[e >> 2] >> (8 * (e & 3)));
}

// e4m3 and back: the conversions of the vector unit, to nearest even; what is above 448 (a quotient's last bit) is 448
__device__ __forceinline__ Eight widen_m(u32x2 w, float scale) {
    Eight r;
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        const auto a = __builtin_amdgcn_cvt_pk_f32_fp8((int)w[k], false), b = __builtin_amdgcn_cvt_pk_f32_fp8((int)w[k], true);
        r.x[4 * k] = a[0] * scale; r.x[4 * k + 1] = a[1] * scale; r.x[4 * k + 2] = b[0] * scale; r.x[4 * k + 3] = b[1] * scale;
    }
    return r;
}
__device__ __forceinline__ float within(float x) { return x != x ? x : fminf(fmaxf(x, -448.0f), 448.0f); }
__device__ __forceinline__ u32x2 narrow_m(const Eight& x) {
    u32x2 w;
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        int c = __builtin_amdgcn_cvt_pk_fp8_f32(within(x.x[4 * k]), within(x.x[4 * k + 1]), 0, false);
        c = __builtin_amdgcn_cvt_pk_fp8_f32(within(x.x[4 * k + 2]), within(x.x[4 * k + 3]), c, true);
        w[k] = (uint32_t)c;
    }
    return w;
}
// v's codes are the upper bits of an fp32 number without its sign: five of exponent (2^-31 .. 1) and three of mantissa
constexpr uint32_t kLowest = (127 - 31) << 3;
__device__ __forceinline__ Eight widen_v(u32x2 w, float scale) {
    Eight r;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const uint32_t c = (w[e >> 2] >> (8 * (e & 3))) & 0xFFu;
        r.x[e] = c ? __uint_as_float((c + kLowest) << 20) * scale : 0.0f;
    }
    return r;
}

// One over a scale and its block's numbers are taken as 2^120 times as large where they are tiny, so that neither is infinite or loses digits
struct Quotient {
    float up, inverse;
    __device__ __forceinline__ Quotient(float largest, float top) {
        up = largest < 0x1p-90f ? 0x1p120f : 1.0f;
        inverse = largest > 0.0f ? top / (largest * up) : 0.0f;
    }
    __device__ __forceinline__ float operator()(float x) const { return (x * up) * inverse; }
};

__device__ __forceinline__ u32x2 narrow_v(const Eight& x, const Quotient& q) {
    u32x2 w = {0, 0};
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const uint32_t u = __float_as_uint(q(x.x[e]));
        const int c = (int)((u + 0x7FFFFu + ((u >> 20) & 1u)) >> 20) - (int)kLowest;
        w[e >> 2] |= (x.x[e] > 0.0f ? (uint32_t)min(max(c, 1), 255) : 0u) << (8 * (e & 3));
    }
    return w;
}

template <bool BITS8>
__global__ __launch_bounds__(kAdamwThreads) void k_adamw(AdamwGroup unused) {
    const auto* g = group_args<AdamwGroup>();
    const uint32_t block = blockIdx.x;
    int k = 0;
#pragma unroll
    for (int i = 1; i < kMaxItems; ++i) k += block >= g->first[i] ? 1 : 0;                 // (those that are not there begin past the last workgroup)
    const auto& item = g->item[k];
    const AdamwStep step = {g->step.one_minus_beta1, g->step.beta1, g->step.one_minus_beta2, g->step.beta2, g->step.inv_c1, g->step.inv_c2, g->step.eps, g->step.rate};
    const float* const scale_at = global_pointer(g->grad_scale);
    const float grad_scale = scale_at ? *scale_at : 1.0f;
    if (!(fabsf(grad_scale) <= 3.402823466e38f)) return;                                  // (the same for all: not finite, nothing is done)
    const int64_t at = (int64_t)(block - g->first[k]) * kAdamwElements + threadIdx.x * 8;
    const int left = (int)min(item.elements - at, (int64_t)8);                            // (none, or fewer: the lanes stay, for the maxima)
    void* const param = global_pointer(item.param);
    const void* const grad = global_pointer(item.grad);
    float* const master = global_pointer(item.master);
    const int dtype = item.dtype, grad_dtype = item.grad_dtype;
    const float rate = step.rate * item.rate_factor, decay = item.decay;
    Eight p, d, m, v;
    if constexpr (BITS8) {
        const int64_t of_scale = left > 0 ? at / kAdamwBlock : 0;
        const float ms = global_pointer(item.m_scale)[of_scale], vs = global_pointer(item.v_scale)[of_scale];
        const u32x2 mw = load_codes(static_cast<const uint8_t*>(global_pointer(item.m)) + at, left), vw = load_codes(static_cast<const uint8_t*>(global_pointer(item.v)) + at, left);
        d = load_any(grad, at, left, grad_dtype);
        p = master ? load_eight<F32>(master + at, left) : load_any(param, at, left, dtype);
        m = widen_m(mw, ms); v = widen_v(vw, vs);
    } else {
        m = load_eight<F32>(static_cast<const float*>(global_pointer(item.m)) + at, left);
        v = load_eight<F32>(static_cast<const float*>(global_pointer(item.v)) + at, left);
        d = load_any(grad, at, left, grad_dtype);
        p = master ? load_eight<F32>(master + at, left) : load_any(param, at, left, dtype);
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const float x = d.x[e] * grad_scale;
        m.x[e] = fmaf(step.beta1, m.x[e], step.one_minus_beta1 * x);
        v.x[e] = fmaf(step.beta2, v.x[e], step.one_minus_beta2 * x * x);
        const float by = m.x[e] * step.inv_c1 / (sqrtf(v.x[e] * step.inv_c2) + step.eps);
        p.x[e] = fmaf(-rate, fmaf(decay, p.x[e], by), p.x[e]);
    }
    if (master) store_eight<F32>(master + at, p, left);
    store_any(param, at, p, left, dtype);
    if constexpr (BITS8) {
        float largest_m = 0.0f, largest_v = 0.0f;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            if (e >= left) { m.x[e] = 0.0f; v.x[e] = 0.0f; }
            largest_m = fmaxf(largest_m, fabsf(m.x[e])); largest_v = fmaxf(largest_v, v.x[e]);
        }
        largest_m = max_of_32(largest_m); largest_v = max_of_32(largest_v);
        const Quotient qm(largest_m, 448.0f), qv(largest_v, 1.875f);
        if ((threadIdx.x & 31) == 0 && left > 0) {
            global_pointer(item.m_scale)[at / kAdamwBlock] = largest_m / 448.0f;
            global_pointer(item.v_scale)[at / kAdamwBlock] = largest_v / 1.875f;
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) m.x[e] = qm(m.x[e]);
        store_codes(static_cast<uint8_t*>(global_pointer(item.m)) + at, narrow_m(m), left);
        store_codes(static_cast<uint8_t*>(global_pointer(item.v)) + at, narrow_v(v, qv), left);
    } else {
        store_eight<F32>(static_cast<float*>(global_pointer(item.m)) + at, m, left);
        store_eight<F32>(static_cast<float*>(global_pointer(item.v)) + at, v, left);
    }
}

hipError_t launch_adamw(const AdamwGroup& g, uint32_t blocks, bool bits8, hipStream_t st) {
    if (bits8) hipLaunchKernelGGL(k_adamw<true>, dim3(blocks), dim3(kAdamwThreads), 0, st, g);
    else hipLaunchKernelGGL(k_adamw<false>, dim3(blocks), dim3(kAdamwThreads), 0, st, g);
    return hipGetLastError();
}

}  // namespace lsp

// One step of AdamW over many tensors in a launch, states in fp32 or in 8 bits.
//
// Bound by memory: a bf16 element takes 22 bytes with states in fp32 (30 with an fp32 master) and 10 with states in 8 bits; nothing is read twice.  A thread
// takes eight elements that follow one another, so that every stream goes in loads of 8 to 32 bytes a lane, and 32 lanes have the 256 elements of a scale:
// its maximum goes through the 32 lanes without LDS.  A workgroup has 2048 elements of one tensor; the tensors' descriptors come with the launch (kMaxItems of
// them), so that a model's many small tensors take few launches and no memory of their own.
#include "adamw.h"
#include "rows.h"

namespace lsp {

// The largest of 32 lanes' numbers in fp64, none of them negative, in all of them: as integers, first the upper halves, then the lower halves of those that have the largest.
// (Lane + 8, 4, 2, 1 of the sixteen, then the other sixteen.)
__device__ __forceinline__ uint32_t top_of_32(uint32_t x) {
    const auto step = [&](int y) { x = max(x, (uint32_t)y); };
    step(__builtin_amdgcn_update_dpp(0, (int)x, 0x128, 0xF, 0xF, false)); step(__builtin_amdgcn_update_dpp(0, (int)x, 0x124, 0xF, 0xF, false));
    step(__builtin_amdgcn_update_dpp(0, (int)x, 0x122, 0xF, 0xF, false)); step(__builtin_amdgcn_update_dpp(0, (int)x, 0x121, 0xF, 0xF, false));
    step(__builtin_amdgcn_ds_swizzle((int)x, 0x401F));
    return x;
}
__device__ __forceinline__ double max_of_32(double x) {
    const uint64_t u = __builtin_bit_cast(uint64_t, x);
    const uint32_t high = top_of_32((uint32_t)(u >> 32)), low = top_of_32((uint32_t)(u >> 32) == high ? (uint32_t)u : 0u);
    return __builtin_bit_cast(double, (uint64_t)high << 32 | low);
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
    uint32_t a = 0, b = 0;
#pragma unroll
    for (int e = 0; e < 7; ++e)
        if (e < left) (e < 4 ? a : b) |= (uint32_t)p[e] << (8 * (e & 3));
    return u32x2{a, b};
}
__device__ __forceinline__ void store_codes(uint8_t* p, u32x2 w, int left) {
    if (left >= 8) { *reinterpret_cast<u32x2*>(p) = w; return; }
#pragma unroll
    for (int e = 0; e < 7; ++e)
        if (e < left) p[e] = (uint8_t)(w[e >> 2] >> (8 * (e & 3)));
}

// States in 8 bits are computed in fp64 up to their rounding, so that what lies near the border between two codes gets the one that the formulas say.  (A product in fp64 takes the
// vector unit no longer than one in fp32.)
struct EightWide { double x[8]; };

// e4m3 and back: the conversions of the vector unit, to nearest even; a quotient above 448, by a last bit, is 448
__device__ __forceinline__ EightWide widen_m(u32x2 w, float scale) {
    EightWide r;
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        const auto a = __builtin_amdgcn_cvt_pk_f32_fp8((int)w[k], false), b = __builtin_amdgcn_cvt_pk_f32_fp8((int)w[k], true);
        r.x[4 * k] = a[0]; r.x[4 * k + 1] = a[1]; r.x[4 * k + 2] = b[0]; r.x[4 * k + 3] = b[1];
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) r.x[e] *= (double)scale;
    return r;
}
__device__ __forceinline__ float within(double x) {
    const float y = (float)x;
    return y != y ? y : fminf(fmaxf(y, -448.0f), 448.0f);
}
__device__ __forceinline__ u32x2 narrow_m(const EightWide& x, double inverse) {
    u32x2 w;
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        int c = __builtin_amdgcn_cvt_pk_fp8_f32(within(x.x[4 * k] * inverse), within(x.x[4 * k + 1] * inverse), 0, false);
        c = __builtin_amdgcn_cvt_pk_fp8_f32(within(x.x[4 * k + 2] * inverse), within(x.x[4 * k + 3] * inverse), c, true);
        w[k] = (uint32_t)c;
    }
    return w;
}
// v's codes are the upper bits of an fp32 number without its sign: five of exponent (2^-31 .. 1) and three of mantissa
constexpr uint32_t kLowest = (127 - 31) << 3;
__device__ __forceinline__ EightWide widen_v(u32x2 w, float scale) {
    EightWide r;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const uint32_t c = (w[e >> 2] >> (8 * (e & 3))) & 0xFFu;
        r.x[e] = (double)(c ? __uint_as_float((c + kLowest) << 20) : 0.0f) * (double)scale;
    }
    return r;
}
__device__ __forceinline__ u32x2 narrow_v(const EightWide& x, double inverse) {
    u32x2 w = {0, 0};
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const uint32_t u = __float_as_uint((float)(x.x[e] * inverse));
        const int c = (int)((u + 0x7FFFFu + ((u >> 20) & 1u)) >> 20) - (int)kLowest;
        w[e >> 2] |= (x.x[e] > 0.0 ? (uint32_t)min(max(c, 1), 255) : 0u) << (8 * (e & 3));
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
    const auto update = [&](float p, float m, float v) {
        const float by = m * step.inv_c1 / (sqrtf(v * step.inv_c2) + step.eps);
        return fmaf(-rate, fmaf(decay, p, by), p);
    };
    const auto load_param = [&] { return master ? load_eight<F32>(master + at, left) : load_any(param, at, left, dtype); };
    const auto store_param = [&](const Eight& p) {
        if (master) store_eight<F32>(master + at, p, left);
        store_any(param, at, p, left, dtype);
    };
    if constexpr (BITS8) {
        uint8_t* const m_at = static_cast<uint8_t*>(global_pointer(item.m)) + at;
        uint8_t* const v_at = static_cast<uint8_t*>(global_pointer(item.v)) + at;
        float* const m_scale = global_pointer(item.m_scale) + (left > 0 ? at / kAdamwBlock : 0);
        float* const v_scale = global_pointer(item.v_scale) + (left > 0 ? at / kAdamwBlock : 0);
        const float ms = *m_scale, vs = *v_scale;
        const u32x2 mw = load_codes(m_at, left), vw = load_codes(v_at, left);
        const Eight d = load_any(grad, at, left, grad_dtype);
        Eight p = load_param();
        EightWide m = widen_m(mw, ms), v = widen_v(vw, vs);
        double top_m = 0.0, top_v = 0.0;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const double x = (double)d.x[e] * (double)grad_scale;
            m.x[e] = g->beta1 * m.x[e] + g->one_minus_beta1 * x;
            v.x[e] = g->beta2 * v.x[e] + g->one_minus_beta2 * x * x;
            p.x[e] = update(p.x[e], (float)m.x[e], (float)v.x[e]);
            if (e < left) { top_m = fmax(top_m, fabs(m.x[e])); top_v = fmax(top_v, v.x[e]); }            // (past a NaN)
        }
        store_param(p);
        top_m = max_of_32(top_m); top_v = max_of_32(top_v);
        if ((threadIdx.x & 31) == 0 && left > 0) { *m_scale = (float)(top_m / 448.0); *v_scale = (float)(top_v / 1.875); }
        store_codes(m_at, narrow_m(m, top_m > 0.0 ? 448.0 / top_m : 0.0), left);
        store_codes(v_at, narrow_v(v, top_v > 0.0 ? 1.875 / top_v : 0.0), left);
    } else {
        float* const m_at = static_cast<float*>(global_pointer(item.m)) + at;
        float* const v_at = static_cast<float*>(global_pointer(item.v)) + at;
        Eight m = load_eight<F32>(m_at, left), v = load_eight<F32>(v_at, left);
        const Eight d = load_any(grad, at, left, grad_dtype);
        Eight p = load_param();
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float x = d.x[e] * grad_scale;
            m.x[e] = fmaf(step.beta1, m.x[e], step.one_minus_beta1 * x);
            v.x[e] = fmaf(step.beta2, v.x[e], step.one_minus_beta2 * x * x);
            p.x[e] = update(p.x[e], m.x[e], v.x[e]);
        }
        store_param(p);
        store_eight<F32>(m_at, m, left);
        store_eight<F32>(v_at, v, left);
    }
}

hipError_t launch_adamw(const AdamwGroup& g, uint32_t blocks, bool bits8, hipStream_t st) {
    if (bits8) hipLaunchKernelGGL(k_adamw<true>, dim3(blocks), dim3(kAdamwThreads), 0, st, g);
    else hipLaunchKernelGGL(k_adamw<false>, dim3(blocks), dim3(kAdamwThreads), 0, st, g);
    return hipGetLastError();
}

}  // namespace lsp

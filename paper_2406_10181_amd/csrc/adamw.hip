// One step of AdamW over many tensors in a launch, states in fp32 or in 8 bits.
//
// Bound by memory: a bf16 element takes 22 bytes with states in fp32 (30 with an fp32 master) and 10 with states in 8 bits; nothing is read twice.  A thread
// takes eight elements that follow one another, so that every stream goes in loads of 8 to 32 bytes a lane, and 32 lanes have the 256 elements of a scale:
// its maximum goes through the 32 lanes without LDS.  A workgroup has 4096 elements of one tensor, in rounds of 2048; the tensors' descriptors come with the launch (52 or
// 64 of them), so that a model's many small tensors take few launches and no memory of their own.
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

// States in 8 bits are computed in fp64 up to their rounding, so that what lies near the border between two codes gets the one that the formulas say.  (A product in fp64, or a
// conversion, takes the vector unit no longer than one in fp32.)
struct EightWide { double x[8]; };

// e4m3: the conversions of the vector unit, to nearest even.  (No quotient is above 448: the largest is 448 (1 + 2^-52) at most, and rounded to fp32 before.)
__device__ __forceinline__ Eight widen_m(u32x2 w) {
    Eight r;
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        const auto a = __builtin_amdgcn_cvt_pk_f32_fp8((int)w[k], false), b = __builtin_amdgcn_cvt_pk_f32_fp8((int)w[k], true);
        r.x[4 * k] = a[0]; r.x[4 * k + 1] = a[1]; r.x[4 * k + 2] = b[0]; r.x[4 * k + 3] = b[1];
    }
    return r;
}
__device__ __forceinline__ u32x2 narrow_m(const EightWide& x, double inverse) {
    u32x2 w;
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        int c = __builtin_amdgcn_cvt_pk_fp8_f32((float)(x.x[4 * k] * inverse), (float)(x.x[4 * k + 1] * inverse), 0, false);
        c = __builtin_amdgcn_cvt_pk_fp8_f32((float)(x.x[4 * k + 2] * inverse), (float)(x.x[4 * k + 3] * inverse), c, true);
        w[k] = (uint32_t)c;
    }
    return w;
}
// v's codes are the upper bits of an fp32 number without its sign: five of exponent (2^-31 .. 1) and three of mantissa
constexpr uint32_t kLowest = (127 - 31) << 3;
__device__ __forceinline__ Eight widen_v(u32x2 w) {
    Eight r;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const uint32_t c = (w[e >> 2] >> (8 * (e & 3))) & 0xFFu;
        r.x[e] = c ? __uint_as_float((c << 20) + (kLowest << 20)) : 0.0f;
    }
    return r;
}
__device__ __forceinline__ u32x2 narrow_v(const EightWide& x, double inverse) {
    u32x2 w = {0, 0};
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const uint32_t u = __float_as_uint((float)(x.x[e] * inverse));
        const int c = (int)(u + ((u >> 20) & 1u) + (0x7FFFFu - (kLowest << 20))) >> 20;
        w[e >> 2] |= min((uint32_t)min(max(c, 1), 255), u) << (8 * (e & 3));                             // (0 stays 0)
    }
    return w;
}

// Where the loads are on their way, and before anything is written, the step is called off if the gradients' scale is not finite.
__device__ __forceinline__ bool finite(float x) { return fabsf(x) <= 3.402823466e38f; }

// m / (sqrt(v) + eps) with the bias corrections in the factors.  QUICK: by the vector unit's square root and reciprocal, each within an ulp; they take what is below 2^-126 for zero, so only
// where eps is 2^-40 or more, which such a root (below 2^-63) does not change.  (bf16, states in 8 bits, 32000 x 4096: 250 us, with quotients as IEEE has them 293.)
template <bool QUICK> __device__ __forceinline__ float updated(float p, float m, float v, const AdamwStep& s, float rate, float rate_decay) {
    p = fmaf(-rate_decay, p, p);
    if constexpr (QUICK) return fmaf(-rate * m, __builtin_amdgcn_rcpf(__builtin_amdgcn_sqrtf(v) + s.eps), p);
    else return fmaf(-rate, m / (sqrtf(v) + s.eps), p);
}

// One over a positive number, 0 of 0: the vector unit's reciprocal (some 2^-26 off) and one step of Newton's, within 2^-50.  (Of states' magnitudes, far from fp64's ends.)
__device__ __forceinline__ double inverse_of(double x) {
    const double r = __builtin_amdgcn_rcp(x);
    return x > 0.0 ? fma(r, fma(-x, r, 1.0), r) : 0.0;
}

// What a workgroup has to know, all of it in scalar registers; pointers to its first element
struct AdamwWork {
    void *param, *m, *v;
    const void* grad;
    float *m_scale, *v_scale, *master;
    AdamwStep step;
    float rate, rate_decay, grad_scale;
    double m_of, v_of, beta1, beta2;
};

// Eight elements of a thread as they lie in memory.  `left`: how many of them there are; the others, and lanes with none, have zeros and go through the maxima with them.
template <typename P, typename G, bool MASTER, bool BITS8> struct Loaded {
    Packed<P> p;
    Packed<G> d;
    Packed<F32> master, m, v;
    u32x2 mw, vw;
    float m_scale, v_scale;
    __device__ __forceinline__ void load(const AdamwWork& w, uint32_t at, int left) {
        d = load_packed<G>(static_cast<const typename G::elem*>(w.grad) + at, left);
        if constexpr (MASTER) master = load_packed<F32>(w.master + at, left);
        else p = load_packed<P>(static_cast<const typename P::elem*>(w.param) + at, left);
        if constexpr (BITS8) {
            mw = load_codes(static_cast<const uint8_t*>(w.m) + at, left);
            vw = load_codes(static_cast<const uint8_t*>(w.v) + at, left);
            const uint32_t of = left > 0 ? at / kAdamwBlock : 0;
            m_scale = w.m_scale[of]; v_scale = w.v_scale[of];
        } else {
            m = load_packed<F32>(static_cast<const float*>(w.m) + at, left);
            v = load_packed<F32>(static_cast<const float*>(w.v) + at, left);
        }
    }
    template <bool QUICK> __device__ __forceinline__ void update(const AdamwWork& w, uint32_t at, int left) const {
        Eight q;
        if constexpr (MASTER) q = widen_eight<F32>(master);
        else q = widen_eight<P>(p);
        const Eight g = widen_eight<G>(d);
        if constexpr (BITS8) {
            const double m_by = w.beta1 * (double)m_scale, v_by = w.beta2 * (double)v_scale;
            const Eight m0 = widen_m(mw), v0 = widen_v(vw);
            EightWide mx, vx;
            double top_m = 0.0, top_v = 0.0;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const double x = (double)g.x[e];
                mx.x[e] = fma(w.m_of, x, m_by * (double)m0.x[e]);
                vx.x[e] = fma(w.v_of * x, x, v_by * (double)v0.x[e]);
                q.x[e] = updated<QUICK>(q.x[e], (float)mx.x[e], (float)vx.x[e], w.step, w.rate, w.rate_decay);
                top_m = fmax(top_m, fabs(mx.x[e])); top_v = fmax(top_v, vx.x[e]);                         // (past a NaN)
            }
            store_param(w, q, at, left);
            top_m = max_of_32(top_m); top_v = max_of_32(top_v);
            if ((threadIdx.x & 31) == 0 && left > 0) { w.m_scale[at / kAdamwBlock] = (float)(top_m * (1.0 / 448.0)); w.v_scale[at / kAdamwBlock] = (float)(top_v * (1.0 / 1.875)); }
            store_codes(static_cast<uint8_t*>(w.m) + at, narrow_m(mx, 448.0 * inverse_of(top_m)), left);
            store_codes(static_cast<uint8_t*>(w.v) + at, narrow_v(vx, 1.875 * inverse_of(top_v)), left);
        } else {
            Eight mx = widen_eight<F32>(m), vx = widen_eight<F32>(v);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float x = g.x[e] * w.grad_scale;
                mx.x[e] = fmaf(w.step.beta1, mx.x[e], w.step.one_minus_beta1 * x);
                vx.x[e] = fmaf(w.step.beta2, vx.x[e], w.step.one_minus_beta2 * x * x);
                q.x[e] = updated<QUICK>(q.x[e], mx.x[e], vx.x[e], w.step, w.rate, w.rate_decay);
            }
            store_param(w, q, at, left);
            store_eight<F32>(static_cast<float*>(w.m) + at, mx, left);
            store_eight<F32>(static_cast<float*>(w.v) + at, vx, left);
        }
    }
    __device__ __forceinline__ static void store_param(const AdamwWork& w, Eight q, uint32_t at, int left) {
        if constexpr (MASTER) {
            store_eight<F32>(w.master + at, q, left);
            // (param is the master rounded: the compiler would round the sum to fp16 without the rounding to fp32 between)
#pragma unroll
            for (int e = 0; e < 8; ++e) asm("" : "+v"(q.x[e]));
        }
        store_eight<P>(static_cast<typename P::elem*>(w.param) + at, q, left);
    }
};

// A workgroup's kAdamwRounds rounds of 2048 elements.  Whole ones are asked for together: more of the memory's latency is behind the arithmetic of others (states in 8 bits, 32000 x 4096
// in bf16: 250 us, one by one 269).
template <typename P, typename G, bool MASTER, bool BITS8, bool QUICK> __device__ __forceinline__ void adamw_of(const AdamwWork& w, int elements) {
    constexpr int kRound = 8 * kAdamwThreads;
    using L = Loaded<P, G, MASTER, BITS8>;
    const uint32_t at = threadIdx.x * 8;
    if (elements >= kAdamwElements) {
        L l[kAdamwRounds];
#pragma unroll
        for (int c = 0; c < kAdamwRounds; ++c) l[c].load(w, at + c * kRound, 8);
        if (!finite(w.grad_scale)) return;
#pragma unroll
        for (int c = 0; c < kAdamwRounds; ++c) {
            if (c) __builtin_amdgcn_sched_barrier(0);
            l[c].template update<QUICK>(w, at + c * kRound, 8);
        }
    } else if (finite(w.grad_scale)) {
        for (int c = 0; c < kAdamwRounds; ++c) {
            const int left = max(min(elements - (int)at - c * kRound, 8), 0);
            L l;
            l.load(w, at + c * kRound, left);
            l.template update<QUICK>(w, at + c * kRound, left);
        }
    }
}
template <typename P, bool BITS8, bool QUICK> __device__ __forceinline__ void adamw_of_grad(const AdamwWork& w, int elements, int grad_dtype) {
    const auto with = [&](auto grad) {
        using G = decltype(grad);
        if (w.master) adamw_of<P, G, true, BITS8, QUICK>(w, elements);
        else adamw_of<P, G, false, BITS8, QUICK>(w, elements);
    };
    if (grad_dtype == LSP_F32) with(F32{});
    else if (grad_dtype == LSP_F16) with(F16{});
    else with(BF16{});
}

// 32000 x 4096 in bf16: states in fp32 528 us, 5.5 TB/s, with an fp32 master 684, 5.75 TB/s; states in 8 bits 250, 5.3 TB/s (moving the same five streams and doing nothing takes 238).
// The tensor is found by a ballot: by a loop over their beginnings in scalar registers 273, for 200 tensors of 4096 elements 25 us instead of 16.
template <bool BITS8, bool QUICK>
__global__ __launch_bounds__(kAdamwThreads, 5) void k_adamw(AdamwGroup<BITS8> unused) {
    const auto* g = group_args<AdamwGroup<BITS8>>();
    const int block = (int)blockIdx.x;
    const int lane = threadIdx.x & 63, begin = g->first[min(lane, AdamwGroup<BITS8>::kItems - 1)];
    const int k = __popcll(__ballot(lane < AdamwGroup<BITS8>::kItems && block >= begin)) - 1;              // (a lane has a tensor: how many begin at this workgroup or before)
    const auto& item = g->item[k];
    AdamwWork w;
    w.step = {g->step.one_minus_beta1, g->step.beta1, g->step.one_minus_beta2, g->step.beta2, g->step.eps, g->step.rate, g->step.decay_rate};
    w.grad_scale = g->grad_scale ? *as_const<float>(g->grad_scale) : 1.0f;
    const int64_t first = (int64_t)(block - g->first[k]) * kAdamwElements;
    const int dtype = (int)(item.elements / kAdamwSizes) & 3, grad_dtype = (int)(item.elements / kAdamwSizes) >> 2;
    const int elements = (int)min(item.elements % kAdamwSizes - first, (int64_t)kAdamwElements), size = dtype == LSP_F32 ? 4 : 2, grad_size = grad_dtype == LSP_F32 ? 4 : 2;
    w.param = global_pointer(static_cast<uint8_t*>(item.param) + first * size);
    w.grad = global_pointer(static_cast<const uint8_t*>(item.grad) + first * grad_size);
    w.m = global_pointer(static_cast<uint8_t*>(item.m) + first * (BITS8 ? 1 : 4));
    w.v = global_pointer(static_cast<uint8_t*>(item.v) + first * (BITS8 ? 1 : 4));
    w.master = item.master ? global_pointer(item.master + first) : nullptr;
    if constexpr (BITS8) {
        w.m_scale = global_pointer(item.m_scale + first / kAdamwBlock);
        w.v_scale = global_pointer(item.v_scale + first / kAdamwBlock);
    }
    w.rate = w.step.rate * item.rate_factor; w.rate_decay = w.step.decay_rate * item.rate_factor * item.decay;
    w.beta1 = g->beta1; w.beta2 = g->beta2;
    w.m_of = g->one_minus_beta1 * (double)w.grad_scale; w.v_of = g->one_minus_beta2 * (double)w.grad_scale * (double)w.grad_scale;
    if (dtype == LSP_F32) adamw_of_grad<F32, BITS8, QUICK>(w, elements, grad_dtype);
    else if (dtype == LSP_F16) adamw_of_grad<F16, BITS8, QUICK>(w, elements, grad_dtype);
    else adamw_of_grad<BF16, BITS8, QUICK>(w, elements, grad_dtype);
}

template <bool BITS8> hipError_t launch_adamw(const AdamwGroup<BITS8>& g, uint32_t blocks, hipStream_t st) {
    if (g.step.eps >= 0x1p-40f) hipLaunchKernelGGL((k_adamw<BITS8, true>), dim3(blocks), dim3(kAdamwThreads), 0, st, g);
    else hipLaunchKernelGGL((k_adamw<BITS8, false>), dim3(blocks), dim3(kAdamwThreads), 0, st, g);
    return hipGetLastError();
}
template hipError_t launch_adamw<false>(const AdamwGroup<false>& g, uint32_t blocks, hipStream_t st);
template hipError_t launch_adamw<true>(const AdamwGroup<true>& g, uint32_t blocks, hipStream_t st);

}  // namespace lsp

// What follows a product before its result is rounded: y = act(p + bias) + residual, in fp32 on the accumulators.
#pragma once
#include "brq_launch.h"
#include "mfma_fp4.h"

namespace brq {

// A kernel's argument for it; empty where the kernel is the product alone.
template <bool EPI>
struct EpilogueArg {};
template <>
struct EpilogueArg<true> { Epilogue e; };

// gelu(t) = t Phi(t), Phi the normal distribution function.  With a = |t|: Q(a) = 1 - Phi(a) = exp(-a^2/2) P(1 / (1 + 0.3 a)), where
// P is the polynomial of degree 8 that is nearest to exp(a^2/2) Q(a) on 0 <= a <= 13.5 in relative error (6e-8), found by weighted
// least squares; Phi(t) = Q(a) for t < 0, 1 - Q(a) else.  The exponential's argument carries 2 roundings, t^2 2^-24 relative in the result;
// 1 / (1 + 0.3 a) and the exponential come from the hardware (1 ulp each).  From t = -13.2 down the exponential is flushed to zero.
__device__ __forceinline__ float gelu_f32(float t) {
    const float a = fabsf(t), s = __builtin_amdgcn_rcpf(__builtin_fmaf(0.3f, a, 1.0f));
    float p = 0.03833479806780815f;
    p = __builtin_fmaf(p, s, -0.1689540594816208f);
    p = __builtin_fmaf(p, s, 0.22822065651416779f);
    p = __builtin_fmaf(p, s, -0.07600235193967819f);
    p = __builtin_fmaf(p, s, 0.142186239361763f);
    p = __builtin_fmaf(p, s, 0.09483278542757034f);
    p = __builtin_fmaf(p, s, 0.12188203632831573f);
    p = __builtin_fmaf(p, s, 0.11949308216571808f);
    p = __builtin_fmaf(p, s, 6.851708349131513e-06f);
    const float q = p * __builtin_amdgcn_exp2f(a * a * -0.72134752044448170f);
    return t * (t < 0.0f ? q : 1.0f - q);
}

template <int N>
__device__ __forceinline__ void activate(float (&v)[N], int act) {      // (uniform)
    if (act == ACT_RELU) {
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = v[i] < 0.0f ? 0.0f : v[i];   // (NaN stays)
    } else if (act == ACT_SILU) {
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = swiglu_f32(v[i], 1.0f);
    } else if (act == ACT_GELU) {
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = gelu_f32(v[i]);
    }
}

__device__ __forceinline__ float residual_at(const Epilogue& e, int64_t row, int64_t col) {
    const uint8_t* p = e.res + row * e.res_pitch;
    return e.res_bf16 ? as_f32((uint32_t)reinterpret_cast<const uint16_t*>(p)[col] << 16) : reinterpret_cast<const float*>(p)[col];
}

}  // namespace brq

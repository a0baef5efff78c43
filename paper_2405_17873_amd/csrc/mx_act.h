// Activations of the microscaled linears, and their slopes, in fp32.
//   gelu       a Phi(a) = max(a, 0) - m Phi(-m), m = |a|, with Phi(-m) = exp(-m^2 / 2) P(t), t = 1 / (1 + 0.29 m), P of degree 6 fitted on [0, 13] to 6.1 10^-7 of
//              the tail up to 2.6 and 8.7 10^-8 m^2 of it behind, about what the exponential's argument carries there.  So negative results keep their relative
//              accuracy down to the smallest normal float32.  (As one exponential of a polynomial on [0, 6], held behind it, bfloat16 results were off by 0.7 %
//              at -7 and 2 % at -13; 16384 x 640 x 5120 geglu took 51 to 57 us, by card, where it takes 55 to 63.)
//   gelu_tanh  a sigma(1.59577 a + 0.0713548 a^3), which is a / 2 (1 + tanh(sqrt(2 / pi) (a + 0.044715 a^3)))
//   silu       a sigma(a)
// Exponential and reciprocal are the hardware's (an ulp each; the argument of the exponential carries 2^-24 of its size).
#pragma once
#include "mx_common.h"

namespace mq {

// sigma(z) of z times -log2(e)
__device__ __forceinline__ float gate_sigma(float z) { return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(z)); }
// (The middle of three: one instruction, where a minimum quiets its operands first.  For NaN it is the lower bound, and the NaN comes back by another factor.)
__device__ __forceinline__ float between(float a, float low, float high) { return __builtin_amdgcn_fmed3f(a, low, high); }
__device__ __forceinline__ float square(float a) { return between(a * a, 0.0f, 1e30f); }  // (finite: products with zero stay zero)
__device__ __forceinline__ float silu_sigma(float a) { return gate_sigma(a * -1.4426950409f); }
__device__ __forceinline__ float tanh_sigma(float a) { return gate_sigma(a * __builtin_fmaf(-0.1029432397f, square(a), -2.3022081985f)); }

// Phi(-m) for m = |a|, and exp(-a^2 / 2).  m is held where that is zero, so that infinite arguments give no infinity times zero.
__device__ __forceinline__ float gelu_size(float a) { return between(fabsf(a), 0.0f, 16.0f); }
__device__ __forceinline__ float gelu_tail(float a, float m, float& gauss) {
    const float t = __builtin_amdgcn_rcpf(__builtin_fmaf(0.29f, m, 1.0f));
    gauss = __builtin_amdgcn_exp2f(a * -0.72134752f * a);
    float p = -0.0958174914f;
    p = __builtin_fmaf(p, t, 0.312764943f);
    p = __builtin_fmaf(p, t, -0.137771845f);
    p = __builtin_fmaf(p, t, 0.215866283f);
    p = __builtin_fmaf(p, t, 0.0849722326f);
    p = __builtin_fmaf(p, t, 0.120265901f);
    p = __builtin_fmaf(p, t, -0.000279949571f);
    return p * gauss;
}
__device__ __forceinline__ float act_gelu(float a) {
    float gauss;
    const float m = gelu_size(a);
    return __builtin_fmaf(-m, gelu_tail(a, m, gauss), between(a, 0.0f, INFINITY));
}
// The activation and its slope.
__device__ __forceinline__ float act_and_slope(float a, int act, float& slope) {
    if (act == MQ_ACT_GELU) {
        float gauss;
        const float m = gelu_size(a), e = gelu_tail(a, m, gauss);
        slope = __builtin_fmaf(a * 0.3989422804f, gauss, a < 0.0f ? e : 1.0f - e);
        return __builtin_fmaf(-m, e, between(a, 0.0f, INFINITY));
    }
    if (act == MQ_ACT_SILU) {
        const float s = silu_sigma(a), f = a * s;
        slope = __builtin_fmaf(f, 1.0f - s, s);
        return f;
    }
    const float s = tanh_sigma(a), f = a * s;
    slope = __builtin_fmaf(f * (1.0f - s), __builtin_fmaf(0.2140644488f, square(a), 1.5957691216f), s);
    return f;
}
// n values; act is the same for the whole wave.
template <int N>
__device__ __forceinline__ void act_values(float* a, int act) {
    if (act == MQ_ACT_NONE) return;
    if (act == MQ_ACT_GELU) {
#pragma unroll
        for (int i = 0; i < N; ++i) a[i] = act_gelu(a[i]);
    } else if (act == MQ_ACT_SILU) {
#pragma unroll
        for (int i = 0; i < N; ++i) a[i] *= silu_sigma(a[i]);
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) a[i] *= tanh_sigma(a[i]);
    }
}

}  // namespace mq

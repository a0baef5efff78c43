// Activations of the microscaled linears, and their slopes, in fp32.
//   gelu       a Phi(a): Phi by erfc(x) = exp(-x^2) t P(t), t = 1 / (1 + 0.33 x), P of degree 7 fitted to 10^-7 of erfc on [0, 10] (5 10^-7 in fp32), so
//              that the tail of negative a keeps its relative accuracy
//   gelu_tanh  a sigma(1.59577 a + 0.0713548 a^3), which is a / 2 (1 + tanh(sqrt(2 / pi) (a + 0.044715 a^3)))
//   silu       a sigma(a)
// Exponential and reciprocal are the hardware's (an ulp each; the argument of the exponential carries 2^-24 of its size).
#pragma once
#include "mx_common.h"

namespace mq {

// sigma(z) of z times -log2(e)
__device__ __forceinline__ float gate_sigma(float z) { return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(z)); }
__device__ __forceinline__ float square(float a) { return fminf(a * a, 1e30f); }  // (finite: products with zero stay zero)
__device__ __forceinline__ float silu_sigma(float a) { return gate_sigma(a * -1.4426950409f); }
__device__ __forceinline__ float tanh_sigma(float a) { return gate_sigma(a * __builtin_fmaf(-0.1029432397f, square(a), -2.3022081985f)); }

// Phi(-|a|) and exp(-a^2 / 2)
__device__ __forceinline__ float gelu_tail(float a, float& gauss) {
    const float m = fabsf(a), t = __builtin_amdgcn_rcpf(__builtin_fmaf(0.23334524f, m, 1.0f));
    gauss = __builtin_amdgcn_exp2f(m * m * -0.72134752f);
    float p = -0.067672479f;
    p = __builtin_fmaf(p, t, 0.23011708f);
    p = __builtin_fmaf(p, t, -0.17557236f);
    p = __builtin_fmaf(p, t, 0.20424775f);
    p = __builtin_fmaf(p, t, 0.023611497f);
    p = __builtin_fmaf(p, t, 0.10061159f);
    p = __builtin_fmaf(p, t, 0.091478027f);
    p = __builtin_fmaf(p, t, 0.093178898f);
    return p * t * gauss;
}
__device__ __forceinline__ float act_gelu(float a) {
    float gauss;
    const float e = gelu_tail(a, gauss);
    return a * (a < 0.0f ? e : 1.0f - e);
}
// The activation and its slope.
__device__ __forceinline__ float act_and_slope(float a, int act, float& slope) {
    if (act == MQ_ACT_GELU) {
        float gauss;
        const float e = gelu_tail(a, gauss), phi = a < 0.0f ? e : 1.0f - e;
        slope = __builtin_fmaf(a * 0.3989422804f, gauss, phi);
        return a * phi;
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

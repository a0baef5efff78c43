// Activations of the microscaled linears, and their slopes, in fp32.
//   gelu       a Phi(a): Phi by erfc(x) = exp(-x^2) t P(t), t = 1 / (1 + 0.33 x), P of degree 7 fitted to 10^-7 of erfc on [0, 10] (5 10^-7 in fp32), so
//              that the tail of negative a keeps its relative accuracy
//   gelu_tanh  a sigma(1.59577 a + 0.0713548 a^3), which is a / 2 (1 + tanh(sqrt(2 / pi) (a + 0.044715 a^3)))
//   silu       a sigma(a)
// Exponential and reciprocal are the hardware's (an ulp each; the argument of the exponential carries 2^-24 of its size).
#pragma once
#include "mx_common.h"

namespace mq {

struct GateTerms {
    float c, d;  // a sigma(c a + d a^3)
};
__device__ __forceinline__ GateTerms gate_terms(int act) { return act == MQ_ACT_SILU ? GateTerms{1.0f, 0.0f} : GateTerms{1.5957691216f, 0.0713548163f}; }

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
__device__ __forceinline__ float gate_sigma(float a, GateTerms g) {
    return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-1.4426950409f * (a * __builtin_fmaf(g.d, a * a, g.c))));
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
    const GateTerms g = gate_terms(act);
    const float s = gate_sigma(a, g), f = a * s;
    slope = __builtin_fmaf(f * (1.0f - s), __builtin_fmaf(3.0f * g.d, a * a, g.c), s);
    return f;
}
// n values; act is the same for the whole wave.
template <int N>
__device__ __forceinline__ void act_values(float* a, int act) {
    if (act == MQ_ACT_NONE) return;
    if (act == MQ_ACT_GELU) {
#pragma unroll
        for (int i = 0; i < N; ++i) a[i] = act_gelu(a[i]);
    } else {
        const GateTerms g = gate_terms(act);
#pragma unroll
        for (int i = 0; i < N; ++i) a[i] *= gate_sigma(a[i], g);
    }
}

}  // namespace mq

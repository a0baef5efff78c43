// Activations of the microscaled linears, and their slopes, in fp32.
//   gelu       a Phi(a) = max(a, 0) - m Phi(-m), m = |a|, with Phi(-m) = 2^(P(m) - m^2 log2(e) / 2), P of degree 7 fitted to the logarithm on [0, 6]: the tail
//              is good to 4 10^-6 of itself.  m is held at 6 in P and in the product, where the result is below 6 10^-9: good to 2 % of itself down to -13.
//              (With a reciprocal and an exponential, good to 5 10^-7, it took nine instructions more: 16384 x 640 x 5120 geglu 62 us where silu takes 40; now 54 and 44.)
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

// Phi(-m) for m = min(|a|, 6) (NaN where a is), with the square of a.
__device__ __forceinline__ float gelu_tail(float a, float m) {
    float p = -1.83481893e-06f;
    p = __builtin_fmaf(p, m, 6.15984318e-05f);
    p = __builtin_fmaf(p, m, -0.000930525886f);
    p = __builtin_fmaf(p, m, 0.00850789435f);
    p = __builtin_fmaf(p, m, -0.0539600737f);
    p = __builtin_fmaf(p, m, 0.262883127f);
    p = __builtin_fmaf(p, m, -1.15125108f);
    p = __builtin_fmaf(p, m, -0.999995291f);
    return __builtin_amdgcn_exp2f(__builtin_fmaf(a * -0.72134752f, a, p));
}
__device__ __forceinline__ float act_gelu(float a) {
    const float m = between(fabsf(a), 0.0f, 6.0f);
    return __builtin_fmaf(-m, gelu_tail(a, m), between(a, 0.0f, INFINITY));
}
// The activation and its slope.
__device__ __forceinline__ float act_and_slope(float a, int act, float& slope) {
    if (act == MQ_ACT_GELU) {
        const float m = between(fabsf(a), 0.0f, 6.0f), e = gelu_tail(a, m), gauss = __builtin_amdgcn_exp2f(a * -0.72134752f * a);
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

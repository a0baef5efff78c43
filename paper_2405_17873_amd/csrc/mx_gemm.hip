// Product of two microscaled 4-bit matrices: Y = A W^T + bias (+ residual), with the MFMAs that take the scales of the blocks as operands.
#include "mx_common.h"

namespace mq {

typedef int int8v __attribute__((ext_vector_type(8)));

// One 32 x 32 x 64 step; S: the byte of the scale words that belongs to it.
template <int S>
__device__ __forceinline__ float16v mx_mfma(int4v w, int4v a, float16v c, int sw, int sa) {
    const int8v W = {w[0], w[1], w[2], w[3], 0, 0, 0, 0}, A = {a[0], a[1], a[2], a[3], 0, 0, 0, 0};
    return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(W, A, c, 4, 4, S, sw, S, sa);
}

// The weights are the MFMA's row operand: a lane then holds, of one row of Y, four runs of four consecutive columns (8 t + 4 h, h the lane's half).
// Two such runs trade places with those of the other half, and the lane has eight consecutive columns, one 16-byte store.
template <int DT>
__device__ __forceinline__ void mx_store_block(const MxGemm& g, const float16v& acc, long m, int n0, int h) {
    if (g.wide) {
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            const int n = n0 + 16 * t + 8 * h;
            const bool on = m < g.M && n < g.N;
            float f[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) f[i] = acc[8 * t + i];
            if (g.res) {
                uint4v r = {0, 0, 0, 0};
                if (on) r = *(const uint4v*)(g.res + m * g.ldr + n);
                // to the accumulators' order: words 0, 1 of both halves are run 2 t, words 2, 3 run 2 t + 1
                const auto p = __builtin_amdgcn_permlane32_swap(r[0], r[2], false, false), q = __builtin_amdgcn_permlane32_swap(r[1], r[3], false, false);
                const uint32_t o[4] = {(uint32_t)p[0], (uint32_t)q[0], (uint32_t)p[1], (uint32_t)q[1]};
#pragma unroll
                for (int i = 0; i < 8; ++i) f[i] += T16<DT>::up((uint16_t)(o[i >> 1] >> (16 * (i & 1))));
            }
            const uint32_t a0 = T16<DT>::pack(f[0], f[1]), a1 = T16<DT>::pack(f[2], f[3]), b0 = T16<DT>::pack(f[4], f[5]), b1 = T16<DT>::pack(f[6], f[7]);
            const auto p = __builtin_amdgcn_permlane32_swap(a0, b0, false, false), q = __builtin_amdgcn_permlane32_swap(a1, b1, false, false);
            if (on) *(uint4v*)(g.y + m * g.ldy + n) = uint4v{(uint32_t)p[0], (uint32_t)q[0], (uint32_t)p[1], (uint32_t)q[1]};
        }
    } else {
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const int n = n0 + 8 * (i >> 2) + 4 * h + (i & 3);
            if (m < g.M && n < g.N) {
                float f = acc[i];
                if (g.res) f += T16<DT>::up(g.res[m * g.ldr + n]);
                g.y[m * g.ldy + n] = T16<DT>::down(f);
            }
        }
    }
}

// The accumulators start from the bias.
template <int DT>
__device__ __forceinline__ float16v mx_bias_block(const MxGemm& g, int n0, int h) {
    float16v c;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        const int n = n0 + 8 * (i >> 2) + 4 * h + (i & 3);
        c[i] = g.bias && n < g.N ? T16<DT>::up(g.bias[n]) : 0.0f;
    }
    return c;
}

// Four waves, a workgroup tile of 128 x 128, operands straight from memory in lane order.
template <int DT>
__global__ __launch_bounds__(256) void mx_gemm_kernel(const MxGemm g) {
    const int lane = threadIdx.x & 63, wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int h = lane >> 5;
    const int ga = blockIdx.x * 4 + (wv & 1) * 2, gw = blockIdx.y * 4 + (wv >> 1) * 2;
    const uint8_t *ac[2], *as[2], *wc[2], *ws[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const long a = ga + i < g.a.groups ? ga + i : g.a.groups - 1, w = gw + i < g.w.groups ? gw + i : g.w.groups - 1;
        ac[i] = g.a.codes + a * g.a.kc * 1024 + lane * 16;
        as[i] = g.a.scales + a * g.a.kq * 256 + lane * 4;
        wc[i] = g.w.codes + w * g.w.kc * 1024 + lane * 16;
        ws[i] = g.w.scales + w * g.w.kq * 256 + lane * 4;
    }
    float16v acc[2][2];
#pragma unroll
    for (int n = 0; n < 2; ++n) {
        const float16v b = mx_bias_block<DT>(g, (gw + n) * 32, h);
        acc[0][n] = b;
        acc[1][n] = b;
    }
    auto step = [&](auto s, int c, const int* sa, const int* sw) {
        int4v a[2], w[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            a[i] = *(const int4v*)(ac[i] + (long)c * 1024);
            w[i] = *(const int4v*)(wc[i] + (long)c * 1024);
        }
#pragma unroll
        for (int m = 0; m < 2; ++m)
#pragma unroll
            for (int n = 0; n < 2; ++n) acc[m][n] = mx_mfma<decltype(s)::value>(w[n], a[m], acc[m][n], sw[n], sa[m]);
    };
    const int kc = g.a.kc;
    for (int q = 0; q < g.a.kq; ++q) {
        int sa[2], sw[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            sa[i] = *(const int*)(as[i] + (long)q * 256);
            sw[i] = *(const int*)(ws[i] + (long)q * 256);
        }
        step(std::integral_constant<int, 0>{}, q * 4, sa, sw);
        if (q * 4 + 1 < kc) step(std::integral_constant<int, 1>{}, q * 4 + 1, sa, sw);
        if (q * 4 + 2 < kc) step(std::integral_constant<int, 2>{}, q * 4 + 2, sa, sw);
        if (q * 4 + 3 < kc) step(std::integral_constant<int, 3>{}, q * 4 + 3, sa, sw);
    }
#pragma unroll
    for (int m = 0; m < 2; ++m)
#pragma unroll
        for (int n = 0; n < 2; ++n) mx_store_block<DT>(g, acc[m][n], (long)(ga + m) * 32 + (lane & 31), (gw + n) * 32, h);
}

int launch_mx_gemm(const MxGemm& g, hipStream_t st) {
    const dim3 grid((unsigned)((g.a.groups + 3) / 4), (unsigned)((g.w.groups + 3) / 4));
    if (g.dtype == MQ_F16)
        mx_gemm_kernel<MQ_F16><<<grid, 256, 0, st>>>(g);
    else
        mx_gemm_kernel<MQ_BF16><<<grid, 256, 0, st>>>(g);
    MQ_HIP_CHECK_LAUNCH();
    return MQ_OK;
}

}  // namespace mq

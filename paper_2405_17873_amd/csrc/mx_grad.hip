// Gradient of a microscaled 4-bit linear with respect to its input: dX = dY W, the 4-bit weights widened to 16 bits on their way into LDS.
#include "mx_common.h"

namespace mq {

typedef short short4v __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) short4v lds_short4v;

struct MxGrad {
    const uint16_t* dy;
    long lddy;
    MxView w;  // weights [N,K]
    const uint8_t* top;
    int M, N, K;
    uint16_t* dx;
    long lddx;
    bool wide_in, wide_out;
};

// The reduction runs over the weights' rows n, along which neither codes nor scales are contiguous: a stage of 64 n x 64 k is widened by its 128
// blocks' threads into LDS as 16-bit rows of k, and read back by the transposing LDS load, which hands a lane consecutive n of one column k.
// Widened weights are taken relative to the largest scale of their block column (top), times 2^SHIFT: fp16 has too few exponents for 2^(s - 127),
// and a value 2^-37 of its column's largest may go.  The product is scaled back at the end, exactly.
template <int DT>
__global__ __launch_bounds__(256) void mx_grad_kernel(const MxGrad g) {
    constexpr int BM = 64, BK = 64, BN = 64;
    constexpr int FIELD = DT == MQ_F16 ? 140 : 125;  // exponent field of a block with the largest scale: 6 units are 49152, or 1.5
    __shared__ __attribute__((aligned(16))) uint8_t wt[BN * BK * 2];
    __shared__ __attribute__((aligned(16))) uint8_t dt[BM * BN * 2];
    const int tid = threadIdx.x, lane = tid & 63, wv = __builtin_amdgcn_readfirstlane(tid >> 6);
    const long m0 = (long)blockIdx.x * BM;
    const int c = blockIdx.y, k0 = c * BK;
    const int wm = wv & 1, wk = wv >> 1;
    float16v acc = {};
    for (int n0 = 0; n0 < g.N; n0 += BN) {
        __syncthreads();
        if (tid < 128) {
            const int grp = tid >> 6, L = tid & 63, j = L & 31, kb = L >> 5, n = grp * 32 + j;
            uint4v v = {0, 0, 0, 0};
            uint32_t s = 0, t = 0;
            if (n0 / 32 + grp < g.w.groups) {
                const long G = n0 / 32 + grp;
                v = *(const uint4v*)(g.w.codes + (G * g.w.kc + c) * 1024 + L * 16);
                s = g.w.scales[(G * g.w.kq + (c >> 2)) * 256 + L * 4 + (c & 3)];
                const int b = c * 2 + kb;
                t = b * 32 < g.K ? g.top[b] : 0;
            }
            const int f = (int)s - (int)t + FIELD;
            const float sc = mx_scale_operand(s == 255u ? 255u : f > 0 ? (uint32_t)f : 0u);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                uint4v o;
                if constexpr (DT == MQ_F16) {
                    o[0] = h2_bits(__builtin_amdgcn_cvt_scalef32_pk_f16_fp4(v[i], sc, 0));
                    o[1] = h2_bits(__builtin_amdgcn_cvt_scalef32_pk_f16_fp4(v[i], sc, 1));
                    o[2] = h2_bits(__builtin_amdgcn_cvt_scalef32_pk_f16_fp4(v[i], sc, 2));
                    o[3] = h2_bits(__builtin_amdgcn_cvt_scalef32_pk_f16_fp4(v[i], sc, 3));
                } else {
                    o[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(v[i], sc, 0));
                    o[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(v[i], sc, 1));
                    o[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(v[i], sc, 2));
                    o[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(v[i], sc, 3));
                }
                *(uint4v*)(wt + n * (BK * 2) + (((kb * 4 + i) ^ (n & 7)) << 4)) = o;
            }
        }
#pragma unroll
        for (int i = 0; i < 2; ++i) {  // dY: 64 rows of 8 pieces
            const int t = i * 256 + tid, r = t >> 3, p = t & 7;
            const int n = n0 + p * 8;
            uint4v v = {0, 0, 0, 0};
            if (m0 + r < g.M && n < g.N) v = load8_16(g.dy + (m0 + r) * g.lddy + n, g.N - n, g.wide_in);
            *(uint4v*)(dt + r * (BN * 2) + ((p ^ (r & 7)) << 4)) = v;
        }
        __syncthreads();
#pragma unroll
        for (int s = 0; s < 4; ++s) {
            const int h = lane >> 5;
            const int r = wm * 32 + (lane & 31), p = s * 2 + h;
            const half8 b = *(const half8*)(dt + r * (BN * 2) + ((p ^ (r & 7)) << 4));
            uint2v a[2];
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                // 16 lanes read 4 rows of 16 columns and get 4 rows of their column
                const int n = s * 16 + h * 8 + u * 4 + ((lane & 15) >> 2);
                const int col = wk * 32 + ((lane >> 4) & 1) * 16 + (lane & 3) * 4;
                const uint32_t at = (uint32_t)(uintptr_t)wt + (uint32_t)(n * (BK * 2) + (((col >> 3) ^ (n & 7)) << 4) + (col & 4) * 2);
                a[u] = __builtin_bit_cast(uint2v, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_short4v*)(uintptr_t)at));
            }
            const uint4v aa = {a[0][0], a[0][1], a[1][0], a[1][1]};
            if constexpr (DT == MQ_F16)
                acc = __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(half8, aa), b, acc, 0, 0, 0);
            else
                acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, aa), __builtin_bit_cast(bf16x8, b), acc, 0, 0, 0);
        }
    }
    const long m = m0 + wm * 32 + (lane & 31);
    const int kcol = k0 + wk * 32, h = lane >> 5;
    if (kcol >= g.K || m >= g.M) return;
    const int back = (int)g.top[kcol >> 5] - FIELD;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        const int k = kcol + 8 * (i >> 2) + 4 * h + (i & 3);
        g.dx[m * g.lddx + k] = T16<DT>::down(ldexpf(acc[i], back));
    }
}

int launch_mx_grad(const void* dy, int M, int N, long lddy, const void* w, const uint8_t* top, int K, void* dx, long lddx, int dtype, hipStream_t st) {
    MxGrad g;
    g.dy = (const uint16_t*)dy;
    g.lddy = lddy;
    g.w = mx_view(w, N, K);
    g.top = top;
    g.M = M;
    g.N = N;
    g.K = K;
    g.dx = (uint16_t*)dx;
    g.lddx = lddx;
    g.wide_in = lddy % 8 == 0 && (uintptr_t)dy % 16 == 0;
    g.wide_out = lddx % 8 == 0 && (uintptr_t)dx % 16 == 0;
    const dim3 grid((unsigned)((M + 63) / 64), (unsigned)g.w.kc);
    if (dtype == MQ_F16)
        mx_grad_kernel<MQ_F16><<<grid, 256, 0, st>>>(g);
    else
        mx_grad_kernel<MQ_BF16><<<grid, 256, 0, st>>>(g);
    MQ_HIP_CHECK_LAUNCH();
    return MQ_OK;
}

}  // namespace mq

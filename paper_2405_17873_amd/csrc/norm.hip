// Layer norm: forward (16-bit output, or straight into microscaled 4-bit floats) and backward.
//
// A row is held in registers by 64 lanes (up to 2048 columns) or by a workgroup (up to 16384), eight consecutive values per lane and step, so that
// it is read once: mean, then the sum of squared deviations from it, then the output.  All sums are taken in fp32.
#include "mx_common.h"

namespace mq {

__device__ __forceinline__ float wave_sum(float v) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
    return v;
}

// Sum over the lanes that share a row.  `slot` (LDS, a workgroup's four waves): unused for 64 lanes.
template <int LPR>
__device__ __forceinline__ float row_sum(float v, float* slot) {
    v = wave_sum(v);
    if constexpr (LPR == 256) {
        const int wv = threadIdx.x >> 6;
        __syncthreads();
        if ((threadIdx.x & 63) == 0) slot[wv] = v;
        __syncthreads();
        v = (slot[0] + slot[1]) + (slot[2] + slot[3]);
    }
    return v;
}

// Eight parameters from column k on, of which n exist.
__device__ __forceinline__ void load_params(const void* p, int dtype, int k, int n, float fill, float* out) {
    if (!p) {
#pragma unroll
        for (int i = 0; i < 8; ++i) out[i] = fill;
    } else if (dtype == MQ_F32) {
        const float* f = (const float*)p + k;
        if (n >= 8 && ((uintptr_t)f & 15) == 0) {
            const float4v a = *(const float4v*)f, b = *(const float4v*)(f + 4);
#pragma unroll
            for (int i = 0; i < 4; ++i) out[i] = a[i], out[4 + i] = b[i];
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) out[i] = i < n ? f[i] : 0.0f;
        }
    } else {
        const uint16_t* h = (const uint16_t*)p + k;
        const uint4v v = load8_16(h, n, ((uintptr_t)h & 15) == 0);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const uint16_t b = (uint16_t)(v[i >> 1] >> (16 * (i & 1)));
            out[i] = dtype == MQ_F16 ? T16<MQ_F16>::up(b) : T16<MQ_BF16>::up(b);
        }
    }
}

template <int DT>
__device__ __forceinline__ void widen8(uint4v v, float* f) {
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] = T16<DT>::up((uint16_t)(v[i >> 1] >> (16 * (i & 1))));
}
template <int DT>
__device__ __forceinline__ uint4v narrow8(const float* f) {
    return uint4v{T16<DT>::pack(f[0], f[1]), T16<DT>::pack(f[2], f[3]), T16<DT>::pack(f[4], f[5]), T16<DT>::pack(f[6], f[7])};
}
__device__ __forceinline__ bool aligned16(const void* p) { return ((uintptr_t)p & 15) == 0; }

template <int DT, int LPR, int VPT, bool MX>
__global__ __launch_bounds__(256) void layer_norm_kernel(const NormArgs g, const int kc, const int kq) {
    __shared__ float slot[4];
    const int li = threadIdx.x % LPR;
    const long row = (long)blockIdx.x * (256 / LPR) + threadIdx.x / LPR;
    const bool real = row < g.M;  // (MX: rows of padding up to a multiple of 32 are written as zeros)
    if (!MX && LPR == 64 && !real) return;
    const uint16_t* x = g.x + row * g.ldx;
    const bool wide = aligned16(x);
    float v[VPT][8];
    float s = 0.0f;
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
        const int k = (i * LPR + li) * 8, n = real ? g.C - k : 0;
        widen8<DT>(n > 0 ? load8_16(x + k, n, wide) : uint4v{0, 0, 0, 0}, v[i]);
#pragma unroll
        for (int e = 0; e < 8; ++e) s += v[i][e];
    }
    const float inv = 1.0f / (float)g.C;
    const float mean = row_sum<LPR>(s, slot) * inv;
    float q = 0.0f;
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
        const int n = g.C - (i * LPR + li) * 8;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            v[i][e] -= mean;
            q += e < n ? v[i][e] * v[i][e] : 0.0f;
        }
    }
    const float rstd = 1.0f / sqrtf(row_sum<LPR>(q, slot) * inv + g.eps);
    if (real && li == 0) {
        if (g.mean) g.mean[row] = mean;
        if (g.rstd) g.rstd[row] = rstd;
    }
    uint16_t* y = MX ? nullptr : g.y + row * g.ldy;
    const bool ywide = aligned16(y);
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
        const int k = (i * LPR + li) * 8, n = g.C - k;
        if (!MX && n <= 0) break;
        float w[8], b[8], o[8];
        if (n > 0) {
            load_params(g.weight, g.param_dtype, k, n, 1.0f, w);
            load_params(g.bias, g.param_dtype, k, n, 0.0f, b);
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) o[e] = n > 0 ? v[i][e] * rstd * w[e] + b[e] : 0.0f;
        if constexpr (!MX) {
            if (real) store8_16(y + k, narrow8<DT>(o), n, ywide);
        } else {
            uint32_t top = 0;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const uint32_t t = __float_as_uint(o[e]) & 0x7FFFFFFFu;
                top = t > top ? t : top;
            }
            const bool in = real && n > 0;  // C % 32 == 0: alike for the four lanes of a block
            top = quad_max(in ? top : 0u);
            const uint32_t sb = mx_scale_byte(top);
            uint32_t codes = mx_codes_f32(o, mx_scale_operand(sb));
            if (!in || sb == 255u) codes = 0;
            const int c = k >> 6, kb = (k >> 5) & 1, part = li & 3;
            const long grp = row >> 5;
            const int L = kb * 32 + (int)(row & 31);
            uint8_t* scales = (uint8_t*)g.mx + ((long)g.M + 31) / 32 * kc * 1024;
            if (c < kc) *(uint32_t*)((uint8_t*)g.mx + (grp * kc + c) * 1024 + L * 16 + part * 4) = codes;
            if (part == 0 && c < kq * 4) scales[(grp * kq + (c >> 2)) * 256 + L * 4 + (c & 3)] = (uint8_t)sb;
        }
    }
}

template <int DT, bool MX>
static int forward(const NormArgs& a, hipStream_t st) {
    const int kc = (a.C + 63) / 64, kq = (kc + 3) / 4;
    // columns that the lanes have to cover: all that exist, or all of the scales' padding
    const int cols = MX ? kq * 256 : a.C;
    const long rows = MX ? ((long)a.M + 31) / 32 * 32 : a.M;
    auto go = [&](auto kernel, int rows_per_wg) { kernel<<<(unsigned)((rows + rows_per_wg - 1) / rows_per_wg), 256, 0, st>>>(a, kc, kq); };
    if (cols <= 512)
        go(layer_norm_kernel<DT, 64, 1, MX>, 4);
    else if (cols <= 1024)
        go(layer_norm_kernel<DT, 64, 2, MX>, 4);
    else if (cols <= 1536)
        go(layer_norm_kernel<DT, 64, 3, MX>, 4);
    else if (cols <= 2048)
        go(layer_norm_kernel<DT, 64, 4, MX>, 4);
    else if (cols <= 4096)
        go(layer_norm_kernel<DT, 256, 2, MX>, 1);
    else if (cols <= 8192)
        go(layer_norm_kernel<DT, 256, 4, MX>, 1);
    else
        go(layer_norm_kernel<DT, 256, 8, MX>, 1);
    MQ_HIP_CHECK_LAUNCH();
    return MQ_OK;
}
int launch_layer_norm(const NormArgs& a, hipStream_t st) { return a.dtype == MQ_F16 ? forward<MQ_F16, false>(a, st) : forward<MQ_BF16, false>(a, st); }
int launch_layer_norm_mx(const NormArgs& a, hipStream_t st) { return a.dtype == MQ_F16 ? forward<MQ_F16, true>(a, st) : forward<MQ_BF16, true>(a, st); }

// Backward.  With xhat = (x - mean) rstd and g = dy weight:  dx = rstd (g - mean(g) - xhat mean(g xhat)) (+ residual);
// dweight = sum over rows of dy xhat, dbias = sum over rows of dy.  A workgroup walks its share of the rows, each lane adding up the columns that it
// holds anyway; the sums of its waves are joined in LDS in wave order and written to the workspace, and a second kernel adds the workgroups' in order:
// the result does not depend on timing.
template <int DT, int LPR, int VPT>
__global__ __launch_bounds__(256) void layer_norm_grad_kernel(const NormArgs g) {
    constexpr int RPW = 256 / LPR;
    extern __shared__ float sums[];  // [2][C] where several rows share a workgroup
    __shared__ float slot[4];
    const int li = threadIdx.x % LPR, ri = threadIdx.x / LPR;
    const float inv = 1.0f / (float)g.C;
    float aw[VPT][8], ab[VPT][8];
#pragma unroll
    for (int i = 0; i < VPT; ++i)
#pragma unroll
        for (int e = 0; e < 8; ++e) aw[i][e] = ab[i][e] = 0.0f;
    for (long row0 = (long)blockIdx.x * RPW; row0 < g.M; row0 += (long)gridDim.x * RPW) {
        const long row = row0 + ri;
        const bool real = row < g.M;
        const float mean = real ? g.mean[row] : 0.0f, rstd = real ? g.rstd[row] : 0.0f;
        const uint16_t *x = g.x + row * g.ldx, *dy = g.dy + row * g.lddy;
        const bool xw = aligned16(x), dw = aligned16(dy);
        float xh[VPT][8], gr[VPT][8];
        float s1 = 0.0f, s2 = 0.0f;
#pragma unroll
        for (int i = 0; i < VPT; ++i) {
            const int k = (i * LPR + li) * 8, n = real ? g.C - k : 0;
            float d[8], w[8];
            widen8<DT>(n > 0 ? load8_16(x + k, n, xw) : uint4v{0, 0, 0, 0}, xh[i]);
            widen8<DT>(n > 0 ? load8_16(dy + k, n, dw) : uint4v{0, 0, 0, 0}, d);
            if (n > 0) load_params(g.weight, g.param_dtype, k, n, 1.0f, w);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                xh[i][e] = e < n ? (xh[i][e] - mean) * rstd : 0.0f;
                gr[i][e] = e < n ? d[e] * w[e] : 0.0f;
                if (e < n) {
                    aw[i][e] += d[e] * xh[i][e];
                    ab[i][e] += d[e];
                }
                s1 += gr[i][e];
                s2 += gr[i][e] * xh[i][e];
            }
        }
        s1 = row_sum<LPR>(s1, slot) * inv;
        s2 = row_sum<LPR>(s2, slot) * inv;
        if (!real) continue;
        uint16_t* dx = g.dx + row * g.lddx;
        const bool ow = aligned16(dx);
        const uint16_t* res = g.res ? g.res + row * g.ldr : nullptr;
        const bool rw = aligned16(res);
#pragma unroll
        for (int i = 0; i < VPT; ++i) {
            const int k = (i * LPR + li) * 8, n = g.C - k;
            if (n <= 0) break;
            float o[8], r[8];
            if (res) widen8<DT>(load8_16(res + k, n, rw), r);
#pragma unroll
            for (int e = 0; e < 8; ++e) o[e] = (gr[i][e] - s1 - xh[i][e] * s2) * rstd + (res ? r[e] : 0.0f);
            store8_16(dx + k, narrow8<DT>(o), n, ow);
        }
    }
    float* out = g.partial + (long)blockIdx.x * 2 * g.C;
    if constexpr (LPR == 64) {
        for (int w = 0; w < RPW; ++w) {
            if (ri == w) {
#pragma unroll
                for (int i = 0; i < VPT; ++i)
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        const int k = (i * LPR + li) * 8 + e;
                        if (k < g.C) {
                            sums[k] = (w ? sums[k] : 0.0f) + aw[i][e];
                            sums[g.C + k] = (w ? sums[g.C + k] : 0.0f) + ab[i][e];
                        }
                    }
            }
            __syncthreads();
        }
        for (int k = threadIdx.x; k < 2 * g.C; k += 256) out[k] = sums[k];
    } else {
#pragma unroll
        for (int i = 0; i < VPT; ++i)
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const int k = (i * LPR + li) * 8 + e;
                if (k < g.C) {
                    out[k] = aw[i][e];
                    out[g.C + k] = ab[i][e];
                }
            }
    }
}

// Adds the workgroups' sums, column by column, in order: 16 runs of them per column side by side.
__global__ __launch_bounds__(256) void layer_norm_join_kernel(const float* partial, int parts, int C, float* dweight, float* dbias) {
    __shared__ float run[16][16];
    const int col = threadIdx.x & 15, r = threadIdx.x >> 4;
    const int k = blockIdx.x * 16 + col;  // of 2 C
    const int per = (parts + 15) / 16, p0 = r * per, p1 = p0 + per < parts ? p0 + per : parts;
    float s = 0.0f;
    if (k < 2 * C)
        for (int p = p0; p < p1; ++p) s += partial[(long)p * 2 * C + k];
    run[r][col] = s;
    __syncthreads();
    if (r == 0 && k < 2 * C) {
        s = run[0][col];
        for (int i = 1; i < 16; ++i) s += run[i][col];
        float* out = k < C ? dweight : dbias;
        if (out) out[k < C ? k : k - C] = s;
    }
}

static int grad_rows_per_wg(long C) { return C <= 2048 ? 4 : 1; }
static long grad_workgroups(long M, long C) {
    const long n = (M + grad_rows_per_wg(C) - 1) / grad_rows_per_wg(C);
    return n < 512 ? n : 512;
}
size_t layer_norm_grad_workspace_bytes(long M, long C) { return (size_t)grad_workgroups(M, C) * 2 * (size_t)C * 4; }

template <int DT>
static int backward(const NormArgs& a, hipStream_t st) {
    const long parts = grad_workgroups(a.M, a.C);
    auto go = [&](auto kernel, size_t lds) { kernel<<<(unsigned)parts, 256, lds, st>>>(a); };
    const size_t lds = (size_t)a.C * 8;
    if (parts > 0) {
        if (a.C <= 512)
            go(layer_norm_grad_kernel<DT, 64, 1>, lds);
        else if (a.C <= 1024)
            go(layer_norm_grad_kernel<DT, 64, 2>, lds);
        else if (a.C <= 1536)
            go(layer_norm_grad_kernel<DT, 64, 3>, lds);
        else if (a.C <= 2048)
            go(layer_norm_grad_kernel<DT, 64, 4>, lds);
        else if (a.C <= 4096)
            go(layer_norm_grad_kernel<DT, 256, 2>, 0);
        else if (a.C <= 8192)
            go(layer_norm_grad_kernel<DT, 256, 4>, 0);
        else
            go(layer_norm_grad_kernel<DT, 256, 8>, 0);
        MQ_HIP_CHECK_LAUNCH();
    }
    if (a.dweight || a.dbias) {
        layer_norm_join_kernel<<<(2 * a.C + 15) / 16, 256, 0, st>>>(a.partial, (int)parts, a.C, a.dweight, a.dbias);
        MQ_HIP_CHECK_LAUNCH();
    }
    return MQ_OK;
}
int launch_layer_norm_grad(const NormArgs& a, hipStream_t st) { return a.dtype == MQ_F16 ? backward<MQ_F16>(a, st) : backward<MQ_BF16>(a, st); }

}  // namespace mq

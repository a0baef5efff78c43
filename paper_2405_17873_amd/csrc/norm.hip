// Layer norm: forward (16-bit output, or straight into microscaled 4-bit floats) and backward.
//
// A row is held in registers by 8, 16, 32 or 64 lanes, so that each has three to five vectors of eight consecutive values (320, 640 and 1280 columns fill
// them without a rest), or by a workgroup (up to 16384 columns), and is read once: mean, then the sum of squared deviations from it, then the output.
// All sums are taken in fp32.  Bound by memory.  us a call among others: forward 16384 x 640 9.0 (4.7 TB/s; 8.0 traced), 2964 x 1280 4.7, 32768 x 2048 43 (6.2
// TB/s), into MXFP4 10.6, 5.4 and 47; backward 18.6 (4.5 TB/s with a residual), 11.8 and 80.  (One row per wave of 64 lanes whatever its length, before stores went through: forward 13.8,
// 6.9, 50, when these took 10.4, 5.5, 41.)
#include <type_traits>

#include "mx_common.h"

namespace mq {

template <int CTRL>
__device__ __forceinline__ float dpp(float v) {
    return __uint_as_float((uint32_t)__builtin_amdgcn_mov_dpp((int)__float_as_uint(v), CTRL, 0xF, 0xF, true));
}
__device__ __forceinline__ float swap_sum16(float v) {
    const auto p = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __uint_as_float((uint32_t)p[0]) + __uint_as_float((uint32_t)p[1]);
}
__device__ __forceinline__ float swap_sum32(float v) {
    const auto p = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __uint_as_float((uint32_t)p[0]) + __uint_as_float((uint32_t)p[1]);
}
// Sum over aligned runs of LANES lanes (8 to 64), the same bits in each of them.
template <int LANES>
__device__ __forceinline__ float lane_sum(float v) {
    v += dpp<0xB1>(v);   // lanes 1,0,3,2 of four
    v += dpp<0x4E>(v);   // lanes 2,3,0,1
    v += dpp<0x141>(v);  // mirror of eight
    if constexpr (LANES >= 16) v += dpp<0x140>(v);  // mirror of sixteen
    if constexpr (LANES >= 32) v = swap_sum16(v);
    if constexpr (LANES >= 64) v = swap_sum32(v);
    return v;
}

// Sum over the lanes that share a row.  `slot` (LDS, one per wave): where that is a workgroup.
template <int LPR>
__device__ __forceinline__ float row_sum(float v, float* slot) {
    v = lane_sum<LPR < 64 ? LPR : 64>(v);
    if constexpr (LPR == 256) {
        __syncthreads();
        if ((threadIdx.x & 63) == 0) slot[threadIdx.x >> 6] = v;
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
        const uint4v v = load8_16(h, n);
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

// A workgroup's rows of a 16-bit matrix.  WIDE (rows on 16-byte boundaries, whole vectors of eight): through a buffer resource, so that what does not exist
// reads as zero and is not written without a branch, and all loads of a row are under way at once.  Otherwise value by value where need be.
template <bool WIDE>
struct Rows {
    const uint16_t* p;
    long ld;
    __amdgpu_buffer_rsrc_t rsrc;
    __device__ __forceinline__ Rows(const uint16_t* base, long ld_, long row0, long rows, int C) : p(base + row0 * ld_), ld(ld_) {
        const long bytes = rows > 0 && base ? ((rows - 1) * ld + C) * 2 : 0;
        if constexpr (WIDE) rsrc = __builtin_amdgcn_make_buffer_rsrc((void*)p, 0, __builtin_amdgcn_readfirstlane((int)bytes), 0x00020000);
    }
    // Eight values from column k of row r (of the workgroup's), of which n exist.
    __device__ __forceinline__ uint4v load(int r, int k, int n) const {
        if constexpr (WIDE) return __builtin_amdgcn_raw_buffer_load_b128(rsrc, n > 0 ? (int)(r * ld + k) * 2 : -16, 0, 0);
        const uint16_t* q = p + r * ld + k;
        return n > 0 ? load8_16(q, n) : uint4v{0, 0, 0, 0};
    }
    __device__ __forceinline__ void store(int r, int k, int n, uint4v v) const {
        if constexpr (WIDE) return __builtin_amdgcn_raw_buffer_store_b128(v, rsrc, n > 0 ? (int)(r * ld + k) * 2 : -16, 0, WRITE_THROUGH);
        uint16_t* q = (uint16_t*)p + r * ld + k;
        if (n > 0) store8_16(q, v, n);
    }
};

// Parameters of VPT vectors of columns, loaded ahead of their use.
template <int VPT, bool WIDE, bool F32>
struct Params {
    uint4v raw[WIDE ? VPT : 1][F32 ? 2 : 1];
    const void* p;
    int dtype;
    __device__ __forceinline__ Params(const void* p_, int dtype_, int C, int LPR, int li) : p(p_), dtype(dtype_) {
        if constexpr (WIDE) {
            const __amdgpu_buffer_rsrc_t r = __builtin_amdgcn_make_buffer_rsrc((void*)p, 0, C * (F32 ? 4 : 2), 0x00020000);
#pragma unroll
            for (int i = 0; i < VPT; ++i)
#pragma unroll
                for (int q = 0; q < (F32 ? 2 : 1); ++q)
                    raw[i][q] = __builtin_amdgcn_raw_buffer_load_b128(r, (i * LPR + li) * (F32 ? 32 : 16) + q * 16, 0, 0);
        }
    }
    template <int DT>
    __device__ __forceinline__ void get(int i, int k, int n, float fill, float* out) const {
        if constexpr (!WIDE) {
            if (n > 0) load_params(p, dtype, k, n, fill, out);
        } else if constexpr (F32) {
#pragma unroll
            for (int e = 0; e < 8; ++e) out[e] = __uint_as_float(raw[i][e >> 2][e & 3]);
        } else {
            widen8<DT>(raw[i][0], out);
        }
    }
};

template <int DT, int LPR, int VPT, bool MX, bool WIDE, bool F32>
__global__ __launch_bounds__(256) void layer_norm_kernel(const NormArgs g, const int kc, const int kq) {
    constexpr int RPW = 256 / LPR;
    __shared__ float slot[4];
    const int li = threadIdx.x % LPR, ri = threadIdx.x / LPR;
    const long row0 = (long)blockIdx.x * RPW, row = row0 + ri;
    const bool real = row < g.M;  // (MX: rows of padding up to a multiple of 32 are written as zeros)
    const long rows = g.M - row0 < RPW ? g.M - row0 : RPW;
    const Rows<WIDE> x(g.x, g.ldx, row0, rows, g.C);
    uint4v raw[VPT];
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
        const int k = (i * LPR + li) * 8;
        raw[i] = x.load(ri, k, real ? g.C - k : 0);
    }
    const Params<VPT, WIDE, F32> weight(g.weight, g.param_dtype, g.C, LPR, li), bias(g.bias, g.param_dtype, g.C, LPR, li);
    float v[VPT][8];
    float s = 0.0f;
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
        widen8<DT>(raw[i], v[i]);
#pragma unroll
        for (int e = 0; e < 8; ++e) s += v[i][e];
    }
    // (Divided, not multiplied by 1 / C: the mean of a row of equal values, whose sum is exact, is then that value, and nothing is left of the row.)
    const float cols = (float)g.C;
    const float mean = row_sum<LPR>(s, slot) / cols;
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
    const float rstd = 1.0f / sqrtf(row_sum<LPR>(q, slot) / cols + g.eps);
    if (real && li == 0) {
        if (g.mean) g.mean[row] = mean;
        if (g.rstd) g.rstd[row] = rstd;
    }
    const long grp = row >> 5;
    auto codes_of = [&](int c, int kb) { return (uint8_t*)g.mx + (grp * kc + c) * 1024 + (kb * 32 + (row & 31)) * 16; };
    auto scale_of = [&](int c, int kb) {
        return (uint8_t*)g.mx + ((long)g.M + 31) / 32 * kc * 1024 + (grp * kq + (c >> 2)) * 256 + (kb * 32 + (row & 31)) * 4 + (c & 3);
    };
    const Rows<WIDE && !MX> y(g.y, g.ldy, row0, rows, g.C);
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
        const int k = (i * LPR + li) * 8, n = g.C - k;
        float w[8], b[8], o[8];
        weight.template get<DT>(i, k, n, 1.0f, w);
        bias.template get<DT>(i, k, n, 0.0f, b);
#pragma unroll
        for (int e = 0; e < 8; ++e) o[e] = n > 0 ? v[i][e] * rstd * w[e] + b[e] : 0.0f;
        if constexpr (!MX) {
            y.store(ri, k, real ? n : 0, narrow8<DT>(o));
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
            if (c < kc) *(uint32_t*)(codes_of(c, kb) + part * 4) = codes;
            if (part == 0 && c < kq * 4) *scale_of(c, kb) = (uint8_t)sb;
        }
    }
    if constexpr (MX) {  // padding that no lane came by
        for (int b = LPR * VPT / 4 + li; b < kq * 8; b += LPR) {
            if (b >> 1 < kc) *(uint4v*)codes_of(b >> 1, b & 1) = uint4v{0, 0, 0, 0};
            *scale_of(b >> 1, b & 1) = 0;
        }
    }
}

// Calls go(lanes per row, vectors per lane) with the form for `vecs` vectors of eight columns.
template <class F>
static void norm_form(int vecs, F go) {
    auto lanes = [&](auto lpr) {
        constexpr int L = decltype(lpr)::value;
        if (vecs <= 3 * L)
            go(lpr, std::integral_constant<int, 3>{});
        else if (vecs <= 4 * L)
            go(lpr, std::integral_constant<int, 4>{});
        else
            go(lpr, std::integral_constant<int, 5>{});
    };
    if (vecs <= 40)
        lanes(std::integral_constant<int, 8>{});
    else if (vecs <= 80)
        lanes(std::integral_constant<int, 16>{});
    else if (vecs <= 160)
        lanes(std::integral_constant<int, 32>{});
    else if (vecs <= 320)
        lanes(std::integral_constant<int, 64>{});
    else if (vecs <= 512)
        go(std::integral_constant<int, 256>{}, std::integral_constant<int, 2>{});
    else if (vecs <= 1280)
        lanes(std::integral_constant<int, 256>{});
    else
        go(std::integral_constant<int, 256>{}, std::integral_constant<int, 8>{});
}

// Whole vectors of eight on 16-byte boundaries, rows of a workgroup within 32-bit offsets; parameters present, fp32 or of the rows' type.
static bool wide_matrix(const void* p, long ld, int M, int C) { return C % 8 == 0 && (M == 1 || ld % 8 == 0) && (uintptr_t)p % 16 == 0 && ld < (1 << 24); }
static bool wide_params(const void* p, const NormArgs& a) { return p && (uintptr_t)p % 16 == 0 && (a.param_dtype == MQ_F32 || a.param_dtype == a.dtype); }

template <int DT, bool MX>
static int forward(const NormArgs& a, hipStream_t st) {
    const int kc = (a.C + 63) / 64, kq = (kc + 3) / 4;
    const long rows = MX ? ((long)a.M + 31) / 32 * 32 : a.M;
    norm_form((a.C + 7) / 8, [&](auto lpr, auto vpt) {
        constexpr int L = decltype(lpr)::value, RPW = 256 / L;
        constexpr int V = decltype(vpt)::value;
        const unsigned grid = (unsigned)((rows + RPW - 1) / RPW);
        const bool wide = wide_matrix(a.x, a.ldx, a.M, a.C) && (MX || wide_matrix(a.y, a.ldy, a.M, a.C)) && wide_params(a.weight, a) && wide_params(a.bias, a);
        if (!wide)
            layer_norm_kernel<DT, L, V, MX, false, false><<<grid, 256, 0, st>>>(a, kc, kq);
        else if (a.param_dtype == MQ_F32)
            layer_norm_kernel<DT, L, V, MX, true, true><<<grid, 256, 0, st>>>(a, kc, kq);
        else
            layer_norm_kernel<DT, L, V, MX, true, false><<<grid, 256, 0, st>>>(a, kc, kq);
    });
    MQ_HIP_CHECK_LAUNCH();
    return MQ_OK;
}
int launch_layer_norm(const NormArgs& a, hipStream_t st) { return a.dtype == MQ_F16 ? forward<MQ_F16, false>(a, st) : forward<MQ_BF16, false>(a, st); }
int launch_layer_norm_mx(const NormArgs& a, hipStream_t st) { return a.dtype == MQ_F16 ? forward<MQ_F16, true>(a, st) : forward<MQ_BF16, true>(a, st); }

// Backward.  With xhat = (x - mean) rstd and g = dy weight:  dx = rstd (g - mean(g) - xhat mean(g xhat)) (+ residual);
// dweight = sum over rows of dy xhat, dbias = sum over rows of dy.  A workgroup walks its share of the rows, each lane adding up the columns that it
// holds anyway; lanes and waves with the same columns are joined in a fixed order and written to the workspace, and a second kernel adds the
// workgroups' in order: the result does not depend on timing.
template <int DT, int LPR, int VPT, bool WIDE, bool F32>
__global__ __launch_bounds__(256) void layer_norm_grad_kernel(const NormArgs g) {
    constexpr int RPW = 256 / LPR, COLS = LPR * VPT * 8;
    __shared__ __attribute__((aligned(16))) float sums[LPR < 256 ? RPW * COLS : 4];  // LPR == 256: for row_sum
    const int li = threadIdx.x % LPR, ri = threadIdx.x / LPR;
    const float cols = (float)g.C;
    float aw[VPT][8], ab[VPT][8];
#pragma unroll
    for (int i = 0; i < VPT; ++i)
#pragma unroll
        for (int e = 0; e < 8; ++e) aw[i][e] = ab[i][e] = 0.0f;
    const Params<VPT, WIDE, F32> weight(g.weight, g.param_dtype, g.C, LPR, li);
    // The rows after these are on their way while these are worked on.
    uint4v rx[VPT], rd[VPT], rr[VPT];
    float mean = 0.0f, rstd = 0.0f;
    auto rows_at = [&](long row0) { return g.M - row0 < RPW ? g.M - row0 : RPW; };
    auto load = [&](long row0) {
        const long rows = rows_at(row0);
        const Rows<WIDE> x(g.x, g.ldx, row0, rows, g.C), dy(g.dy, g.lddy, row0, rows, g.C);
        const bool real = ri < rows;
#pragma unroll
        for (int i = 0; i < VPT; ++i) {
            const int k = (i * LPR + li) * 8, n = real ? g.C - k : 0;
            rx[i] = x.load(ri, k, n);
            rd[i] = dy.load(ri, k, n);
        }
        mean = real ? g.mean[row0 + ri] : 0.0f;
        rstd = real ? g.rstd[row0 + ri] : 0.0f;
    };
    auto load_residual = [&](long row0) {
        if (!g.res) return;
        const long rows = rows_at(row0);
        const Rows<WIDE> res(g.res, g.ldr, row0, rows, g.C);
#pragma unroll
        for (int i = 0; i < VPT; ++i) {
            const int k = (i * LPR + li) * 8;
            rr[i] = res.load(ri, k, ri < rows ? g.C - k : 0);
        }
    };
    const long stride = (long)gridDim.x * RPW;
    long row0 = (long)blockIdx.x * RPW;
    if (WIDE) load(row0), load_residual(row0);
    for (; row0 < g.M; row0 += stride) {
        if (!WIDE) load(row0), load_residual(row0);  // (pieces of vectors take too many registers to have two rows of)
        const float m = mean, r = rstd;
        float xh[VPT][8], gr[VPT][8];
        float s1 = 0.0f, s2 = 0.0f;
#pragma unroll
        for (int i = 0; i < VPT; ++i) {
            const int k = (i * LPR + li) * 8, n = g.C - k;
            float d[8], w[8];
            widen8<DT>(rx[i], xh[i]);
            widen8<DT>(rd[i], d);  // zero where there is no value
            weight.template get<DT>(i, k, n, 1.0f, w);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                xh[i][e] = (WIDE ? n > 0 : e < n) ? (xh[i][e] - m) * r : 0.0f;  // (a far mean over a small variance passes fp32's range)
                gr[i][e] = WIDE || e < n ? d[e] * w[e] : 0.0f;
                aw[i][e] += d[e] * xh[i][e];
                ab[i][e] += d[e];
                s1 += gr[i][e];
                s2 += gr[i][e] * xh[i][e];
            }
        }
        if (WIDE && row0 + stride < g.M) load(row0 + stride);
        s1 = row_sum<LPR>(s1, sums) / cols;
        s2 = row_sum<LPR>(s2, sums) / cols;
        const long rows = rows_at(row0);
        const Rows<WIDE> dx(g.dx, g.lddx, row0, rows, g.C);
#pragma unroll
        for (int i = 0; i < VPT; ++i) {
            const int k = (i * LPR + li) * 8, n = g.C - k;
            float o[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) o[e] = (gr[i][e] - s1 - xh[i][e] * s2) * r;
            if (g.res) {
                float a[8];
                widen8<DT>(rr[i], a);
#pragma unroll
                for (int e = 0; e < 8; ++e) o[e] += a[e];
            }
            dx.store(ri, k, ri < rows ? n : 0, narrow8<DT>(o));
        }
        if (WIDE && row0 + stride < g.M) load_residual(row0 + stride);
    }
    float* out = g.partial + (long)blockIdx.x * 2 * g.C;
#pragma unroll
    for (int which = 0; which < 2; ++which) {  // one of the two sums after the other: the rows' sums of a column lie below one another
        const float(&acc)[VPT][8] = which ? ab : aw;
        if constexpr (LPR < 256) {
            __syncthreads();
#pragma unroll
            for (int i = 0; i < VPT; ++i)
#pragma unroll
                for (int q = 0; q < 2; ++q)
                    *(float4v*)(sums + ri * COLS + (i * LPR + li) * 8 + q * 4) = float4v{acc[i][4 * q], acc[i][4 * q + 1], acc[i][4 * q + 2], acc[i][4 * q + 3]};
            __syncthreads();
            for (int k = threadIdx.x; k < g.C; k += 256) {
                float v = sums[k];
#pragma unroll
                for (int j = 1; j < RPW; ++j) v += sums[j * COLS + k];
                out[which * g.C + k] = v;
            }
        } else {
#pragma unroll
            for (int i = 0; i < VPT; ++i)
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const int k = (i * LPR + li) * 8 + e;
                    if (k < g.C) out[which * g.C + k] = acc[i][e];
                }
        }
    }
}

// Adds the workgroups' sums, column by column, in order: 32 columns per workgroup, and 32 runs of parts side by side.
__global__ __launch_bounds__(256) void layer_norm_join_kernel(const float* partial, int parts, int C, float* dweight, float* dbias) {
    __shared__ float run[32][33];
    const int col = threadIdx.x & 7, r = threadIdx.x >> 3;
    const int k = blockIdx.x * 32 + col * 4;  // of 2 C
    const int per = (parts + 31) / 32, p0 = r * per, p1 = p0 + per < parts ? p0 + per : parts;
    float s[4] = {0.0f, 0.0f, 0.0f, 0.0f};
    if (k + 4 <= 2 * C && C % 2 == 0) {
#pragma unroll 8
        for (int p = p0; p < p1; ++p) {
            const float4v v = *(const float4v*)(partial + (long)p * 2 * C + k);
#pragma unroll
            for (int e = 0; e < 4; ++e) s[e] += v[e];
        }
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (k + e < 2 * C)
                for (int p = p0; p < p1; ++p) s[e] += partial[(long)p * 2 * C + k + e];
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) run[r][col * 4 + e] = s[e];
    __syncthreads();
    const int j = blockIdx.x * 32 + threadIdx.x;
    if (threadIdx.x < 32 && j < 2 * C) {
        float t = run[0][threadIdx.x];
#pragma unroll
        for (int i = 1; i < 32; ++i) t += run[i][threadIdx.x];
        float* out = j < C ? dweight : dbias;
        if (out) out[j < C ? j : j - C] = t;
    }
}

// Rows that a workgroup has in registers at a time, and the number of workgroups: one per compute unit (a wave's registers leave room for one, and the
// sums of two would only be more to join; us, 256 / 512 workgroups: 16384 x 640 20.1 / 24.5, 2964 x 1280 11.5 / 15.4, 32768 x 2048 81.6 / 83.5).
static int grad_rows_per_wg(long C) {
    const long v = (C + 7) / 8;
    return v <= 40 ? 32 : v <= 80 ? 16 : v <= 160 ? 8 : v <= 320 ? 4 : 1;
}
static long grad_workgroups(long M, long C) {
    const long n = (M + grad_rows_per_wg(C) - 1) / grad_rows_per_wg(C);
    return n < 256 ? n : 256;
}
size_t layer_norm_grad_workspace_bytes(long M, long C) { return (size_t)grad_workgroups(M, C) * 2 * (size_t)C * 4; }

template <int DT>
static int backward(const NormArgs& a, hipStream_t st) {
    const long parts = grad_workgroups(a.M, a.C);
    if (parts > 0) {
        norm_form((a.C + 7) / 8, [&](auto lpr, auto vpt) {
            constexpr int L = decltype(lpr)::value, V = decltype(vpt)::value;
            const bool wide = wide_matrix(a.x, a.ldx, a.M, a.C) && wide_matrix(a.dy, a.lddy, a.M, a.C) && wide_matrix(a.dx, a.lddx, a.M, a.C) &&
                              (!a.res || wide_matrix(a.res, a.ldr, a.M, a.C)) && wide_params(a.weight, a);
            if (!wide)
                layer_norm_grad_kernel<DT, L, V, false, false><<<(unsigned)parts, 256, 0, st>>>(a);
            else if (a.param_dtype == MQ_F32)
                layer_norm_grad_kernel<DT, L, V, true, true><<<(unsigned)parts, 256, 0, st>>>(a);
            else
                layer_norm_grad_kernel<DT, L, V, true, false><<<(unsigned)parts, 256, 0, st>>>(a);
        });
        MQ_HIP_CHECK_LAUNCH();
    }
    if (a.dweight || a.dbias) {
        layer_norm_join_kernel<<<(2 * a.C + 31) / 32, 256, 0, st>>>(a.partial, (int)parts, a.C, a.dweight, a.dbias);
        MQ_HIP_CHECK_LAUNCH();
    }
    return MQ_OK;
}
int launch_layer_norm_grad(const NormArgs& a, hipStream_t st) { return a.dtype == MQ_F16 ? backward<MQ_F16>(a, st) : backward<MQ_BF16>(a, st); }

}  // namespace mq

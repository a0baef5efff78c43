// Product of few rows with a microscaled 4-bit weight matrix, where reading the weights is what counts.
//
// A workgroup has 32 columns of Y and eight waves, each with a part of the reduction, whose sums are joined in LDS in wave order.  A lane's operand of a
// 32x32x64 MFMA is one block of 32 consecutive values of one row: 16-bit activations are quantised right into the operand, without a lane knowing of any
// other, and one launch does the whole linear.
#pragma once
#include "mx_act.h"

namespace mq {

typedef int int8v __attribute__((ext_vector_type(8)));

struct MxRows {
    MxGemm g;
    const uint16_t* x;  // 16-bit activations, or null: g.a
    long ldx;
};

// KIND: MX_ACT, MX_GATED.  Gated: half of the waves have the values' columns, the other half the gates'.
template <int DT, bool MXIN, int RG, int U, int KIND>
__global__ __launch_bounds__(512, 1) void mx_rows_kernel(const MxRows r) {
    constexpr bool ACT = KIND & MX_ACT, GATED = KIND & MX_GATED;
    const MxGemm& g = r.g;
    constexpr int NW = GATED ? 4 : 8, ROW = 32 + 4;  // waves to a column; of sums in LDS, in floats
    constexpr bool QUAD = MXIN && U == 4;  // steps of whole scale words
    extern __shared__ __attribute__((aligned(16))) float sums[];  // [NW][RG * 32][ROW]
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wv = wave % NW;
    const int h = lane >> 5, j = lane & 31;
    const int kc = g.w.kc, kq = g.w.kq, outs = GATED ? g.N >> 1 : g.N;
    const int gw = GATED ? blockIdx.x + wave / NW * (g.w.groups >> 1) : blockIdx.x;
    const int c0 = QUAD ? kq * wv / NW * 4 : kc * wv / NW;
    const int c1 = QUAD ? (kq * (wv + 1) / NW * 4 < kc ? kq * (wv + 1) / NW * 4 : kc) : kc * (wv + 1) / NW;
    const uint8_t *wc = g.w.codes + (long)gw * kc * 1024 + lane * 16, *ws = g.w.scales + (long)gw * kq * 256 + lane * 4;
    float16v acc[RG];
#pragma unroll
    for (int m = 0; m < RG; ++m)
#pragma unroll
        for (int i = 0; i < 16; ++i) acc[m][i] = 0.0f;

    for (int c = c0; c < c1; c += U) {
        int4v w[U];
        int sw[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int cc = c + u < c1 ? c + u : c1 - 1;
            w[u] = *(const int4v*)(wc + (long)cc * 1024);
            sw[u] = QUAD && u ? sw[0] : *(const int*)(ws + (cc >> 2) * 256);
        }
        int4v a[U][RG];
        int sa[U][RG];
        if constexpr (MXIN) {
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int cc = c + u < c1 ? c + u : c1 - 1;
#pragma unroll
                for (int m = 0; m < RG; ++m) {
                    const long grp = m < g.a.groups ? m : g.a.groups - 1;
                    a[u][m] = *(const int4v*)(g.a.codes + (grp * kc + cc) * 1024 + lane * 16);
                    sa[u][m] = QUAD && u ? sa[0][m] : *(const int*)(g.a.scales + (grp * kq + (cc >> 2)) * 256 + lane * 4);
                }
            }
        } else {
            uint4v v[U][RG][4];
#pragma unroll
            for (int u = 0; u < U; ++u)
#pragma unroll
                for (int m = 0; m < RG; ++m) {
                    const int k = (c + u) * 64 + h * 32;
                    const bool in = m * 32 + j < g.M && c + u < c1 && k < g.K;
                    const uint16_t* p = r.x + (m * 32 + j) * r.ldx + k;
#pragma unroll
                    for (int i = 0; i < 4; ++i) v[u][m][i] = in ? load8_16(p + i * 8, 8) : uint4v{0, 0, 0, 0};
                }
#pragma unroll
            for (int u = 0; u < U; ++u)
#pragma unroll
                for (int m = 0; m < RG; ++m) {
                    uint32_t top = 0;
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const uint32_t t = mx_top_16<DT>(v[u][m][i]);
                        top = t > top ? t : top;
                    }
                    sa[u][m] = (int)mx_scale_byte(top);
                    const float s = mx_scale_operand((uint32_t)sa[u][m]);
#pragma unroll
                    for (int i = 0; i < 4; ++i) a[u][m][i] = (int)mx_codes_16<DT>(v[u][m][i], s);
                }
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (c + u < c1) {
                const int byte = 8 * (QUAD ? u : (c + u) & 3);
#pragma unroll
                for (int m = 0; m < RG; ++m) {
                    const int8v W = {w[u][0], w[u][1], w[u][2], w[u][3], 0, 0, 0, 0};
                    const int8v A = {a[u][m][0], a[u][m][1], a[u][m][2], a[u][m][3], 0, 0, 0, 0};
                    acc[m] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(W, A, acc[m], 4, 4, 0, sw[u] >> byte, 0, MXIN ? sa[u][m] >> byte : sa[u][m]);
                }
            }
        }
    }
    // a lane holds, of one row, runs of four columns
#pragma unroll
    for (int m = 0; m < RG; ++m) {
        if (m * 32 + j < g.M) {
            float* p = sums + (wave * RG * 32 + m * 32 + j) * ROW + 4 * h;
#pragma unroll
            for (int t = 0; t < 4; ++t) *(float4v*)(p + 8 * t) = float4v{acc[m][4 * t], acc[m][4 * t + 1], acc[m][4 * t + 2], acc[m][4 * t + 3]};
        }
    }
    __syncthreads();
    for (int i = threadIdx.x; i < g.M * 4; i += 512) {  // runs of eight columns
        const int m = i >> 2, q = i & 3, n = blockIdx.x * 32 + q * 8, left = outs - n;
        if (left <= 0) continue;
        float f[8], gate[8];
        // The sums of one half's columns, with their bias.
        auto total = [&](int part, float* f) {
#pragma unroll
            for (int e = 0; e < 8; ++e) f[e] = 0.0f;
#pragma unroll
            for (int w = 0; w < NW; ++w) {
                const float* p = sums + ((part * NW + w) * RG * 32 + m) * ROW + q * 8;
                const float4v lo = *(const float4v*)p, hi = *(const float4v*)(p + 4);
#pragma unroll
                for (int e = 0; e < 4; ++e) f[e] += lo[e], f[4 + e] += hi[e];
            }
            if (g.bias) {
                const uint4v b = load8_16(g.bias + part * outs + n, left);
#pragma unroll
                for (int e = 0; e < 8; ++e) f[e] += T16<DT>::up((uint16_t)(b[e >> 1] >> (16 * (e & 1))));
            }
        };
        auto store = [&](uint16_t* p, const float* f) {
            store8_16(p, uint4v{T16<DT>::pack(f[0], f[1]), T16<DT>::pack(f[2], f[3]), T16<DT>::pack(f[4], f[5]), T16<DT>::pack(f[6], f[7])}, left);
        };
        const long row = m;
        total(0, f);
        if constexpr (GATED) total(1, gate);
        if constexpr (ACT) {
            if (g.pre) {
                store(g.pre + row * g.ldpre + n, f);
                if constexpr (GATED) store(g.pre + row * g.ldpre + outs + n, gate);
            }
            if constexpr (GATED) {
                act_values<8>(gate, g.act);
#pragma unroll
                for (int e = 0; e < 8; ++e) f[e] *= gate[e];
            } else {
                act_values<8>(f, g.act);
            }
        }
        if (g.res) {
            const uint4v b = load8_16(g.res + row * g.ldr + n, left);
#pragma unroll
            for (int e = 0; e < 8; ++e) f[e] += T16<DT>::up((uint16_t)(b[e >> 1] >> (16 * (e & 1))));
        }
        store(g.y + row * g.ldy + n, f);
    }
}

template <int DT, bool MXIN, int RG, int U, int KIND>
static int run_mx_rows(const MxRows& r, hipStream_t st) {
    constexpr int BYTES = 8 * RG * 32 * (32 + 4) * 4;
    auto kernel = mx_rows_kernel<DT, MXIN, RG, U, KIND>;
    static PerDevice prepared;
    if (const int rc = allow_lds(prepared, (const void*)kernel, BYTES)) return rc;
    kernel<<<(unsigned)((KIND & MX_GATED) ? r.g.w.groups / 2 : r.g.w.groups), 512, BYTES, st>>>(r);
    MQ_HIP_CHECK_LAUNCH();
    return MQ_OK;
}

}  // namespace mq

// Product of few rows with a microscaled 4-bit weight matrix, where reading the weights is what counts.
//
// A workgroup has 32 columns of Y and eight waves, each with a part of the reduction, whose sums are joined in LDS in wave order.  A lane's operand of a
// 32x32x64 MFMA is one block of 32 consecutive values of one row: 16-bit activations are quantised right into the operand, without a lane knowing of any
// other, and one launch does the whole linear.
#include "mx_common.h"

namespace mq {

typedef int int8v __attribute__((ext_vector_type(8)));

struct MxRows {
    MxGemm g;
    const uint16_t* x;  // 16-bit activations, or null: g.a
    long ldx;
};

template <int DT, bool MXIN, int RG, int U>
__global__ __launch_bounds__(512, 1) void mx_rows_kernel(const MxRows r) {
    const MxGemm& g = r.g;
    constexpr int NW = 8, ROW = 32 + 4;  // of sums in LDS, in floats
    constexpr bool QUAD = MXIN && U == 4;  // steps of whole scale words
    extern __shared__ __attribute__((aligned(16))) float sums[];  // [NW][RG * 32][ROW]
    const int lane = threadIdx.x & 63, wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int h = lane >> 5, j = lane & 31;
    const int kc = g.w.kc, kq = g.w.kq, gw = blockIdx.x;
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
            float* p = sums + (wv * RG * 32 + m * 32 + j) * ROW + 4 * h;
#pragma unroll
            for (int t = 0; t < 4; ++t) *(float4v*)(p + 8 * t) = float4v{acc[m][4 * t], acc[m][4 * t + 1], acc[m][4 * t + 2], acc[m][4 * t + 3]};
        }
    }
    __syncthreads();
    for (int i = threadIdx.x; i < g.M * 4; i += 512) {  // runs of eight columns
        const int m = i >> 2, q = i & 3, n = gw * 32 + q * 8, left = g.N - n;
        if (left <= 0) continue;
        float f[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) f[e] = 0.0f;
#pragma unroll
        for (int w = 0; w < NW; ++w) {
            const float* p = sums + (w * RG * 32 + m) * ROW + q * 8;
            const float4v lo = *(const float4v*)p, hi = *(const float4v*)(p + 4);
#pragma unroll
            for (int e = 0; e < 4; ++e) f[e] += lo[e], f[4 + e] += hi[e];
        }
        if (g.bias) {
            const uint4v b = load8_16(g.bias + n, left);
#pragma unroll
            for (int e = 0; e < 8; ++e) f[e] += T16<DT>::up((uint16_t)(b[e >> 1] >> (16 * (e & 1))));
        }
        if (g.res) {
            const uint16_t* p = g.res + m * g.ldr + n;
            const uint4v b = load8_16(p, left);
#pragma unroll
            for (int e = 0; e < 8; ++e) f[e] += T16<DT>::up((uint16_t)(b[e >> 1] >> (16 * (e & 1))));
        }
        uint16_t* y = g.y + m * g.ldy + n;
        store8_16(y, uint4v{T16<DT>::pack(f[0], f[1]), T16<DT>::pack(f[2], f[3]), T16<DT>::pack(f[4], f[5]), T16<DT>::pack(f[6], f[7])}, left);
    }
}

template <int DT, bool MXIN, int RG, int U>
static int run_mx_rows(const MxRows& r, hipStream_t st) {
    constexpr int BYTES = 8 * RG * 32 * (32 + 4) * 4;
    auto kernel = mx_rows_kernel<DT, MXIN, RG, U>;
    static PerDevice prepared;
    if (const int rc = allow_lds(prepared, (const void*)kernel, BYTES)) return rc;
    kernel<<<(unsigned)r.g.w.groups, 512, BYTES, st>>>(r);
    MQ_HIP_CHECK_LAUNCH();
    return MQ_OK;
}

// us, steps of two 64-k tiles / of a scale word (four tiles): 8 x 1280 x 10240 3.9 / 4.4, 16 x 8192 x 2048 5.7 / 4.9, 8 x 5120 x 20480 (334 MB of
// weights in turn) 16.5 / 15.0, 3.7 TB/s; 48 x 2048 x 640 4.4 / 5.3, 64 x 5120 x 5120 6.9 / 8.2.
template <int DT>
static int choose_mx_rows(const MxRows& r, hipStream_t st) {
    if (r.x) return run_mx_rows<DT, false, 1, 2>(r, st);
    if (r.g.M > 64) return run_mx_rows<DT, true, 4, 4>(r, st);
    if (r.g.M > 32) return run_mx_rows<DT, true, 2, 2>(r, st);
    return r.g.w.kq >= 16 ? run_mx_rows<DT, true, 1, 4>(r, st) : run_mx_rows<DT, true, 1, 2>(r, st);
}

// Whether this kernel takes a product: up to 64 rows always, up to 128 where tiles of 128 x 128 would leave most of the chip idle.  us, this / tiles:
// 64 x 1280 x 10240 4.9 / 6.6, 77 x 2048 x 640 4.7 / 7.7, 128 x 5120 x 5120 8.2 / 14.7; 100 x 1280 x 10240 8.0 / 7.0, 100 x 5120 x 20480 32 / 21.
bool mx_rows_takes(int M, int N) { return M <= 64 || (M <= 128 && N <= 256 * 32); }
// Whether it also quantises: every workgroup then reads and converts all activations.  us, in the kernel / before it: 1 x 320 x 1280 3.5 / 5.3, 8 x 1280 x
// 10240 6.1 / 6.5, 32 x 1280 x 1280 5.6 / 6.2; 1 x 5120 x 20480 21.0 / 19.3, 16 x 8192 x 2048 12.8 / 10.0, 48 x 2048 x 640 9.8 / 9.1.
bool mx_rows_quantizes(int M, int N, int K) { return M <= 32 && (long)M * K * ((N + 31) / 32) <= 2500000; }

int launch_mx_rows(const MxGemm& g, const void* x, long ldx, hipStream_t st) {
    MxRows r;
    r.g = g;
    r.x = (const uint16_t*)x;
    r.ldx = ldx;
    return g.dtype == MQ_F16 ? choose_mx_rows<MQ_F16>(r, st) : choose_mx_rows<MQ_BF16>(r, st);
}

}  // namespace mq

// Products of few rows with microscaled 4-bit weights, with an activation or a gate behind them, of one matrix or by expert: one launch.
#include "mx_act.h"

namespace mq {

typedef int int8v __attribute__((ext_vector_type(8)));

// A workgroup has 32 columns of Y (gated: and their gates', in the second half of the waves) and the rows of one expert (blockIdx.y; without offsets all of them),
// 32 at a time.  Of a slab of 2048 k (with four waves 1024), all threads quantise the rows into LDS as the MFMAs want them, while each wave's weights, 256 k (gated 512), are on their way
// to its registers; the waves' sums are joined in LDS in wave order.
// Bound by the weights.  32 rows of 32 experts, 2048 x 2560 each (bfloat16, gated, 45 MB for the experts that have rows) 10.8 us (18.5 with the rows quantised by every
// wave for itself, two steps of 64 k in flight).
template <int DT, bool GATED, int WAVES>
__global__ __launch_bounds__(WAVES * 64, 4) void mx_few_rows_kernel(const MxGemm g, const uint16_t* x, const long ldx) {
    constexpr int PARTS = GATED ? 2 : 1, NW = WAVES / PARTS, ROW = 32 + 4;  // NW: waves to a column; ROW: of sums, in floats
    constexpr int SLAB = WAVES * 4, TILES = SLAB / NW;  // in tiles of 64 k; TILES: a wave's
    constexpr int CODES = SLAB * 1024, SCALES = SLAB / 4 * 256, SUMS = WAVES * 32 * ROW * 4;
    __shared__ __attribute__((aligned(16))) uint8_t lds[CODES + SCALES > SUMS ? CODES + SCALES : SUMS];
    const int e = blockIdx.y;
    int first = g.offsets ? g.offsets[e] : 0, end = g.offsets ? g.offsets[e + 1] : g.M;
    first = __builtin_amdgcn_readfirstlane(first < 0 ? 0 : first);
    end = __builtin_amdgcn_readfirstlane(end > g.M ? g.M : end);
    if (first >= end) return;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wv = wave % NW, h = lane >> 5, j = lane & 31;
    const int kc = g.w.kc, kq = g.w.kq, outs = GATED ? g.N >> 1 : g.N;
    const uint16_t* bias = g.bias ? g.bias + (long)e * g.N : nullptr;
    const long group = (long)e * g.w.groups + (wave / NW) * (g.w.groups >> 1) + blockIdx.x;
    const uint8_t *codes = g.w.codes + group * kc * 1024 + lane * 16, *scales = g.w.scales + group * kq * 256 + lane * 4;
    float* sums = (float*)lds;
    bool used = false;
    for (; first < end; first += 32) {
        const int rows = end - first < 32 ? end - first : 32;
        float16v acc;
#pragma unroll
        for (int i = 0; i < 16; ++i) acc[i] = 0.0f;
        for (int slab = 0; slab < kc; slab += SLAB) {
            const int c = slab + wv * TILES;
            int4v w[TILES];
            int sw[TILES / 4];
            if (c < kc) {
#pragma unroll
                for (int i = 0; i < TILES; ++i) {
                    const int at = c + i < kc ? c + i : kc - 1;
                    w[i] = *(const int4v*)(codes + (long)at * 1024);
                    if (i % 4 == 0) sw[i / 4] = *(const int*)(scales + (at >> 2) * 256);
                }
            }
            if (used) __syncthreads();  // (the last slab, or the last rows' sums, are read)
            used = true;
            const int blocks = (kc - slab < SLAB ? kc - slab : SLAB) * 2;
#pragma unroll 1
            for (int i = threadIdx.x; i < rows * SLAB * 2; i += WAVES * 64) {
                const int row = i / (SLAB * 2), b = i % (SLAB * 2), k = slab * 64 + b * 32;
                if (b >= blocks) continue;
                uint4v v[4];
                const uint16_t* from = x + (first + row) * ldx + k;
#pragma unroll
                for (int u = 0; u < 4; ++u) v[u] = k < g.K ? load8_16(from + u * 8, 8) : uint4v{0, 0, 0, 0};
                uint32_t top = 0;
#pragma unroll
                for (int u = 0; u < 4; ++u) {
                    const uint32_t t = mx_top_16<DT>(v[u]);
                    top = t > top ? t : top;
                }
                const uint32_t s = mx_scale_byte(top);
                const float scale = mx_scale_operand(s);
                const int at = (b & 1) * 32 + row;
                *(uint4v*)(lds + (b >> 1) * 1024 + at * 16) =
                    uint4v{mx_codes_16<DT>(v[0], scale), mx_codes_16<DT>(v[1], scale), mx_codes_16<DT>(v[2], scale), mx_codes_16<DT>(v[3], scale)};
                lds[CODES + (b >> 3) * 256 + at * 4 + ((b >> 1) & 3)] = (uint8_t)s;
            }
            __syncthreads();
#pragma unroll
            for (int i = 0; i < TILES; ++i) {
                if (c + i < kc) {
                    const int4v a = *(const int4v*)(lds + (wv * TILES + i) * 1024 + lane * 16);
                    const int sa = *(const int*)(lds + CODES + (wv * TILES + i) / 4 * 256 + lane * 4);
                    const int8v A = {a[0], a[1], a[2], a[3], 0, 0, 0, 0}, W = {w[i][0], w[i][1], w[i][2], w[i][3], 0, 0, 0, 0};
                    acc = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(W, A, acc, 4, 4, 0, sw[i / 4] >> (8 * (i % 4)), 0, sa >> (8 * (i % 4)));
                }
            }
        }
        __syncthreads();
        if (j < rows) {
            float* to = sums + (wave * 32 + j) * ROW + 4 * h;
#pragma unroll
            for (int t = 0; t < 4; ++t) *(float4v*)(to + 8 * t) = float4v{acc[4 * t], acc[4 * t + 1], acc[4 * t + 2], acc[4 * t + 3]};
        }
        __syncthreads();
        // runs of eight columns of a row, a thread each
        const int m = threadIdx.x >> 2, q = threadIdx.x & 3, n = blockIdx.x * 32 + q * 8, left = outs - n;
        float f[PARTS][8];
        if (m < rows && left > 0) {
#pragma unroll
            for (int p = 0; p < PARTS; ++p) {
#pragma unroll
                for (int i = 0; i < 8; ++i) f[p][i] = 0.0f;
#pragma unroll
                for (int w = 0; w < NW; ++w) {
                    const float* from = sums + ((p * NW + w) * 32 + m) * ROW + q * 8;
                    const float4v lo = *(const float4v*)from, hi = *(const float4v*)(from + 4);
#pragma unroll
                    for (int i = 0; i < 4; ++i) f[p][i] += lo[i], f[p][4 + i] += hi[i];
                }
                if (bias) {
                    const uint4v b = load8_16(bias + p * outs + n, left);
#pragma unroll
                    for (int i = 0; i < 8; ++i) f[p][i] += T16<DT>::up((uint16_t)(b[i >> 1] >> (16 * (i & 1))));
                }
            }
        }
        if (m < rows && left > 0) {
            auto store = [&](uint16_t* to, const float* v) {
                store8_16(to, uint4v{T16<DT>::pack(v[0], v[1]), T16<DT>::pack(v[2], v[3]), T16<DT>::pack(v[4], v[5]), T16<DT>::pack(v[6], v[7])}, left);
            };
            const long row = first + m;
            if (g.pre) {
#pragma unroll
                for (int p = 0; p < PARTS; ++p) store(g.pre + row * g.ldpre + p * outs + n, f[p]);
            }
            act_values<8>(f[PARTS - 1], g.act);
            if constexpr (GATED) {
#pragma unroll
                for (int i = 0; i < 8; ++i) f[0][i] *= f[1][i];
            }
            if (g.res) {
                const uint4v b = load8_16(g.res + row * g.ldr + n, left);
#pragma unroll
                for (int i = 0; i < 8; ++i) f[0][i] += T16<DT>::up((uint16_t)(b[i >> 1] >> (16 * (i & 1))));
            }
            store(g.y + row * g.ldy + n, f[0]);
        }
    }
}

template <int DT, bool GATED, int WAVES>
static int run_mx_few_rows(const MxGemm& g, const void* x, long ldx, hipStream_t st) {
    const dim3 grid((unsigned)(GATED ? g.w.groups / 2 : g.w.groups), (unsigned)(g.offsets ? g.experts : 1));
    mx_few_rows_kernel<DT, GATED, WAVES><<<grid, WAVES * 64, 0, st>>>(g, (const uint16_t*)x, ldx);
    MQ_HIP_CHECK_LAUNCH();
    return MQ_OK;
}
// Eight waves, or four without a gate by expert, where there are workgroups enough.  us, eight / four: 32 rows of 32 experts, 2048 x 2560, 13.9 / 12.2, 128 of 64,
// 2880 x 2880, 52 / 43; gated 13.0 / 12.8 and, of 5760, 79 / 80; one matrix, 8 x 1280 x 5120, 4.8 / 5.3, 32 x 2048 x 2560 gated 7.0 / 8.8.
template <int DT>
static int choose_mx_few_rows(const MxGemm& g, bool gated, const void* x, long ldx, hipStream_t st) {
    if (gated) return run_mx_few_rows<DT, true, 8>(g, x, ldx, st);
    return g.offsets ? run_mx_few_rows<DT, false, 4>(g, x, ldx, st) : run_mx_few_rows<DT, false, 8>(g, x, ldx, st);
}
int launch_mx_few_rows(const MxGemm& g, bool gated, const void* x, long ldx, hipStream_t st) {
    return g.dtype == MQ_F16 ? choose_mx_few_rows<MQ_F16>(g, gated, x, ldx, st) : choose_mx_few_rows<MQ_BF16>(g, gated, x, ldx, st);
}

// Whether one launch takes the product of a matrix: little work to quantise, or one slab.  us, one launch / quantised before it: 8 x 1280 x 10240 gated 5.5 / 7.9,
// 32 x 2048 x 2560 gated 6.9 / 8.3, 32 x 1280 x 10240 gated 7.2 / 7.9; 8 x 5120 x 20480 19.5 / 16.4, 16 x 8192 x 2048 12.2 / 9.2.  (Against every wave quantising for
// itself: 8 x 1280 x 5120 4.8 / 5.7, 3 x 6944 x 256 gated 8.2 / 16.8, 1 x 320 x 1280 3.5 / 3.2.)  Linears without an activation have the kernel in which every wave does: it is
// ahead with short reductions, 1 x 320 x 1280 3.0 where this one, without an activation, takes 3.4, 16 x 320 x 320 3.2 / 4.3, 32 x 640 x 640 4.1 / 5.4, and behind with others, 8 x 1280 x
// 1280 4.4 / 3.9, 8 x 1280 x 5120 4.5 / 4.0, 24 x 2048 x 1280 5.9 / 5.1, 2 x 6944 x 256 9.1 / 6.2.
bool mx_few_rows_takes(int M, int N, int K) { return M <= 32 && (K <= 2048 || mx_rows_quantizes(M, N, K)); }

}  // namespace mq

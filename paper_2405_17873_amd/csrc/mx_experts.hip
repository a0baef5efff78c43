// Products of rows sorted by expert with each expert's microscaled 4-bit weights.
//
// Only the GPU knows how many rows an expert has.  Few rows: a workgroup per expert and 32 columns, which leaves at once where there are none.  Otherwise
// all rows are quantised as one matrix, a plan lists the row tiles, and a launch of workgroups as many as the chip holds walks over them.  The
// matrix' groups of 32 rows are not the experts': a tile starts with the whole group that holds the expert's first row, and leaves the other experts' rows of
// it alone.
#include "expert_walk.h"
#include "mx_gemm_core.h"

namespace mq {

// The quantisation of all rows, and in the launch's first workgroup the plan: a wave has 64 experts at a time.
template <int DT>
__global__ __launch_bounds__(256) void mx_quantize_plan_kernel(const uint16_t* x, int M, int K, long ldx, uint8_t* codes, uint8_t* scales, int kc, int kq, const int* offsets,
                                                               int experts, int tile_rows, MxRowPlan* plan) {
    if (blockIdx.y == 0) {
        if (blockIdx.x > 0 || blockIdx.z > 0 || threadIdx.x >= 64) return;
        ExpertWalk walk;
        for (; walk.base < experts; walk.next()) {
            walk.load(offsets, experts, M, tile_rows, 31);
            const int at = walk.before + walk.upto - walk.count;
            for (int i = 0; i < walk.count; ++i) plan->tile[at + i] = MxPlanTile{walk.base + (int)threadIdx.x, walk.start + i * tile_rows, walk.first, walk.end};
        }
        if (threadIdx.x == 0) plan->tiles = (uint32_t)walk.before;
        return;
    }
    mx_quantize_groups<DT>(x, M, K, ldx, codes, scales, kc, kq, (int)blockIdx.y - 1 + blockIdx.z * 65534L, blockIdx.x);
}

typedef int int8v __attribute__((ext_vector_type(8)));

// Few rows of an expert: a workgroup has 32 columns of Y (gated: and their gates', in the second half of the waves) and the expert's rows, 32 at a time.  Of a slab
// of 2048 k, all threads quantise the rows into LDS as the MFMAs want them, while each wave's weights, 256 k (gated 512), are on their way to its registers; the
// waves' sums are joined in LDS in wave order.
// Bound by the weights.  32 rows of 32 experts, 2048 x 2560 each (bfloat16, gated, 45 MB for the experts that have rows): 18.5 us with the rows quantised by
// every wave for itself, two steps of 64 k in flight.
template <int DT, bool GATED>
__global__ __launch_bounds__(512, 4) void mx_experts_rows_kernel(const MxGemm g, const uint16_t* x, const long ldx) {
    constexpr int PARTS = GATED ? 2 : 1, NW = 8 / PARTS, ROW = 32 + 4;  // NW: waves to a column; ROW: of sums, in floats
    constexpr int SLAB = 32, TILES = SLAB / NW;  // in tiles of 64 k; TILES: a wave's
    constexpr int CODES = SLAB * 1024, SCALES = SLAB / 4 * 256, SUMS = 8 * 32 * ROW * 4;
    __shared__ __attribute__((aligned(16))) uint8_t lds[CODES + SCALES > SUMS ? CODES + SCALES : SUMS];
    const int e = blockIdx.y;
    int first = g.offsets[e], end = g.offsets[e + 1];
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
            for (int i = threadIdx.x; i < rows * 64; i += 512) {
                const int row = i >> 6, b = i & 63, k = slab * 64 + b * 32;
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
        const int m = threadIdx.x >> 2, q = threadIdx.x & 3, n = blockIdx.x * 32 + q * 8;
        float f[PARTS][8];
        if (m < rows) {
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
                    const uint4v b = load8_16(bias + p * outs + n, 8);
#pragma unroll
                    for (int i = 0; i < 8; ++i) f[p][i] += T16<DT>::up((uint16_t)(b[i >> 1] >> (16 * (i & 1))));
                }
            }
        }
        if (m < rows) {  // (columns are whole blocks of 32)
            auto store = [&](uint16_t* to, const float* v) {
                store8_16(to, uint4v{T16<DT>::pack(v[0], v[1]), T16<DT>::pack(v[2], v[3]), T16<DT>::pack(v[4], v[5]), T16<DT>::pack(v[6], v[7])}, 8);
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
            store(g.y + row * g.ldy + n, f[0]);
        }
    }
}

// Whether a workgroup per expert and 32 columns takes the product: few rows to an expert.
static bool mx_experts_rows(long M, int experts) { return M <= 8L * experts || M <= 32; }

size_t mx_experts_workspace_bytes(long M, long N, long K, int experts) {
    return mx_experts_rows(M, experts) ? 0 : mx_plan_bytes(M, experts, 128) + up256(mx_bytes(M, K));
}

template <int DT, int KIND>
static int choose_mx_experts(MxGemm g, const void* x, long ldx, void* ws, hipStream_t st) {
    if (mx_experts_rows(g.M, g.experts)) {
        constexpr bool GATED = KIND & MX_GATED;
        mx_experts_rows_kernel<DT, GATED><<<dim3((unsigned)(GATED ? g.w.groups / 2 : g.w.groups), (unsigned)g.experts), 512, 0, st>>>(g, (const uint16_t*)x, ldx);
        MQ_HIP_CHECK_LAUNCH();
        return MQ_OK;
    }
    MxRowPlan* plan = (MxRowPlan*)ws;
    void* a = (char*)ws + mx_plan_bytes(g.M, g.experts, 128);
    g.a = mx_view(a, g.M, g.K);
    g.plan = plan;
    const bool odd = !mx_wide(g.y, g.ldy) || (g.pre && !mx_wide(g.pre, g.ldpre)) || (uintptr_t)g.bias % 16 != 0;
    constexpr long CUS = 256;
    // us (bfloat16, gated, with the quantisation), tiles of 256 x 256 / 128 x 128: 16384 rows of 8 even experts, 2048 x 8192 158 / 193, uneven ones 171 / 207, of one 155 / 191;
    // 4096 of 4, 2048 x 4096 40 / 34, 4001 of 16, 1280 x 2048 (fp16, no gate) 23 / 20.  Bands of 4 row tiles / of 8, each in the faster tiles: 158 / 177, 171 / 181, 155 / 155,
    // 33.6 / 33.8, 19.9 / 20.1.
    const bool large = !odd && g.M / g.experts >= 512 && ((g.a.groups + 7L) / 8) * ((g.w.groups + 7L) / 8) >= 2 * CUS;
    const int rows = large ? 256 : 128;
    const long most = 65534;  // groups in one plane of the grid, behind the plan's row of it
    const dim3 grid((unsigned)g.a.kq, (unsigned)((g.a.groups < most ? g.a.groups : most) + 1), (unsigned)((g.a.groups + most - 1) / most));
    mx_quantize_plan_kernel<DT><<<grid, 256, 0, st>>>((const uint16_t*)x, g.M, g.K, ldx, (uint8_t*)g.a.codes, (uint8_t*)g.a.scales, g.a.kc, g.a.kq, g.offsets, g.experts,
                                                      rows, plan);
    MQ_HIP_CHECK_LAUNCH();
    const long bound = mx_plan_bound(g.M, g.experts, rows);
    if (odd) return run_mx_form<DT, MX_ODD, KIND, 2, 2, 2, 2, 4>(g, 8, 1L << 31, bound, st);
    return large ? run_mx_form<DT, MX_PLAIN, KIND, 2, 4, 4, 2, 4>(g, 4, CUS, bound, st) : run_mx_form<DT, MX_PLAIN, KIND, 2, 2, 2, 2, 4>(g, 4, 2 * CUS, bound, st);
}

int launch_mx_experts(const MxGemm& g, bool gated, const void* x, long ldx, void* ws, hipStream_t st) {
    constexpr int ONE = MX_ACT | MX_EXPERTS, TWO = MX_ACT | MX_GATED | MX_EXPERTS;
    if (g.dtype == MQ_F16) return gated ? choose_mx_experts<MQ_F16, TWO>(g, x, ldx, ws, st) : choose_mx_experts<MQ_F16, ONE>(g, x, ldx, ws, st);
    return gated ? choose_mx_experts<MQ_BF16, TWO>(g, x, ldx, ws, st) : choose_mx_experts<MQ_BF16, ONE>(g, x, ldx, ws, st);
}

}  // namespace mq

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

// Few rows of an expert: see mx_few_rows_kernel.  us (bfloat16), that / tiles, for 4, 8, 16 and 32 rows to an expert (uneven): 32 experts of 2048 x 2560, gated 17 / 19, 21 / 22,
// 28 / 23, 42 / 24; 8 of 2048 x 4096, gated 11.0 / 13.0 (8 rows), 13.2 / 13.9, 18.9 / 14.1; 64 of 1280 x 1280 15.0 / 17.1, 17.7 / 17.2, 25.7 / 17.7.  (Few experts with a long
// reduction would turn earlier: 64 rows of 4, 6400 x 1408, 23.0 / 21.5.)  The host does not know how uneven the rows are.  With all of them one expert's it passes over them 32 at a time,
// reading the weights again: 256 rows of 32 experts, 2048 x 2560, gated 37 (even 21; one row more, and so in tiles, 12 and 23), 512 of 64, 1280 x 1280, 67 (17; 11 and 18),
// 32768 of 4096, 128 x 128, 4360 (41; 59 and 97).
static bool mx_experts_rows(long M, int experts) { return M <= 8L * experts || M <= 32; }

size_t mx_experts_workspace_bytes(long M, long N, long K, int experts) {
    return mx_experts_rows(M, experts) ? 0 : mx_plan_bytes(M, experts, 128) + up256(mx_bytes(M, K));
}

template <int DT, int KIND>
static int choose_mx_experts(MxGemm g, const void* x, long ldx, void* ws, hipStream_t st) {
    if (mx_experts_rows(g.M, g.experts)) return launch_mx_few_rows(g, KIND & MX_GATED, x, ldx, st);
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

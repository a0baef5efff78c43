// Products of rows sorted by expert with each expert's microscaled 4-bit weights.
//
// Only the GPU knows how many rows an expert has.  Few rows: a workgroup per expert and 32 columns, which leaves at once where there are none.  Otherwise
// all rows are quantised as one matrix, a plan lists the row tiles, and a launch of workgroups as many as the chip holds walks over them.  The
// matrix' groups of 32 rows are not the experts': a tile starts with the whole group that holds the expert's first row, and leaves the other experts' rows of
// it alone.
#include "mx_gemm_core.h"
#include "mx_rows_core.h"

namespace mq {

// One workgroup; thread e has experts e, e + 256, ...  `below`: 31 for tiles that start with whole groups, or 0.  Offsets that fall, or leave 0 .. M, are held at what came before.
__global__ __launch_bounds__(256) void mx_plan_kernel(const int* offsets, int experts, int M, int tile_rows, int below, MxRowPlan* plan) {
    __shared__ int top[256], count[256];
    int reach = 0, tiles = 0;  // of all the experts of the turns before
    for (int e0 = 0; e0 < experts; e0 += 256) {
        const int e = e0 + (int)threadIdx.x;
        int first = e < experts ? offsets[e] : 0, end = e < experts ? offsets[e + 1] : 0;
        first = first < 0 ? 0 : first > M ? M : first;
        end = end < 0 ? 0 : end > M ? M : end;
        // the furthest end in front of this expert
        __syncthreads();
        top[threadIdx.x] = end;
        __syncthreads();
        for (int d = 1; d < 256; d <<= 1) {
            const int o = (int)threadIdx.x >= d ? top[threadIdx.x - d] : 0;
            __syncthreads();
            if (o > top[threadIdx.x]) top[threadIdx.x] = o;
            __syncthreads();
        }
        int before = threadIdx.x ? top[threadIdx.x - 1] : 0;
        before = before > reach ? before : reach;
        first = first > before ? first : before;
        const int start = first & ~below, n = e < experts && end > first ? (end - start + tile_rows - 1) / tile_rows : 0;
        count[threadIdx.x] = n;
        __syncthreads();
        for (int d = 1; d < 256; d <<= 1) {
            const int o = (int)threadIdx.x >= d ? count[threadIdx.x - d] : 0;
            __syncthreads();
            count[threadIdx.x] += o;
            __syncthreads();
        }
        const int at = tiles + count[threadIdx.x] - n;
        for (int i = 0; i < n; ++i) plan->tile[at + i] = MxPlanTile{e, start + i * tile_rows, first, end};
        tiles += count[255];
        reach = top[255] > reach ? top[255] : reach;
    }
    if (threadIdx.x == 0) plan->tiles = (uint32_t)tiles;
}

int launch_mx_plan(const int* offsets, int experts, int M, int tile_rows, bool whole_groups, MxRowPlan* plan, hipStream_t st) {
    mx_plan_kernel<<<1, 256, 0, st>>>(offsets, experts, M, tile_rows, whole_groups ? 31 : 0, plan);
    MQ_HIP_CHECK_LAUNCH();
    return MQ_OK;
}

// Whether a workgroup per expert and 32 columns takes the product: few rows to an expert.
static bool mx_experts_rows(long M, int experts) { return M <= 8L * experts || M <= 32; }

size_t mx_experts_workspace_bytes(long M, long N, long K, int experts) {
    return mx_experts_rows(M, experts) ? 0 : mx_plan_bytes(M, experts, 128) + up256(mx_bytes(M, K));
}

template <int DT, int KIND>
static int choose_mx_experts(MxGemm g, const void* x, long ldx, void* ws, hipStream_t st) {
    if (mx_experts_rows(g.M, g.experts)) {
        MxRows r;
        r.g = g;
        r.x = (const uint16_t*)x;
        r.ldx = ldx;
        return run_mx_rows<DT, false, 1, 2, KIND>(r, st);
    }
    MxRowPlan* plan = (MxRowPlan*)ws;
    void* a = (char*)ws + mx_plan_bytes(g.M, g.experts, 128);
    if (const int rc = launch_mx_quantize(x, g.M, g.K, ldx, g.dtype, a, st)) return rc;
    g.a = mx_view(a, g.M, g.K);
    g.plan = plan;
    const bool odd = !mx_wide(g.y, g.ldy) || (g.pre && !mx_wide(g.pre, g.ldpre)) || (uintptr_t)g.bias % 16 != 0;
    constexpr long CUS = 256;
    const bool large = !odd && g.M / g.experts >= 512 && ((g.a.groups + 7L) / 8) * ((g.w.groups + 7L) / 8) >= 2 * CUS;
    const int rows = large ? 256 : 128;
    if (const int rc = launch_mx_plan(g.offsets, g.experts, g.M, rows, true, plan, st)) return rc;
    const long bound = mx_plan_bound(g.M, g.experts, rows);
    if (odd) return run_mx_form<DT, MX_ODD, KIND, 2, 2, 2, 2, 4>(g, 8, 1L << 31, bound, st);
    return large ? run_mx_form<DT, MX_PLAIN, KIND, 2, 4, 4, 2, 4>(g, 8, CUS, bound, st) : run_mx_form<DT, MX_PLAIN, KIND, 2, 2, 2, 2, 4>(g, 8, 2 * CUS, bound, st);
}

int launch_mx_experts(const MxGemm& g, bool gated, const void* x, long ldx, void* ws, hipStream_t st) {
    constexpr int ONE = MX_ACT | MX_EXPERTS, TWO = MX_ACT | MX_GATED | MX_EXPERTS;
    if (g.dtype == MQ_F16) return gated ? choose_mx_experts<MQ_F16, TWO>(g, x, ldx, ws, st) : choose_mx_experts<MQ_F16, ONE>(g, x, ldx, ws, st);
    return gated ? choose_mx_experts<MQ_BF16, TWO>(g, x, ldx, ws, st) : choose_mx_experts<MQ_BF16, ONE>(g, x, ldx, ws, st);
}

}  // namespace mq

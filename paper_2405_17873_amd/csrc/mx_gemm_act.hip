// Products of microscaled 4-bit matrices with an activation or a gate behind them.
#include "mx_gemm_core.h"

namespace mq {

template <int DT, int WM, int WN, int TM, int TN, int S>
static int run_mx_act(const MxGemm& g, bool gated, bool odd, long band, long most, hipStream_t st) {
    if (odd)
        return gated ? run_mx_form<DT, MX_ODD, MX_ACT | MX_GATED, 2, 2, 2, 2, 4>(g, band, 1L << 31, 0, st)
                     : run_mx_form<DT, MX_ODD, MX_ACT, 2, 2, 2, 2, 4>(g, band, 1L << 31, 0, st);
    if (gated) return run_mx_form<DT, MX_PLAIN, MX_ACT | MX_GATED, WM, WN, TM, TN, S>(g, band, most, 0, st);
    return g.res ? run_mx_form<DT, MX_RES, MX_ACT, WM, WN, TM, TN, S>(g, band, most, 0, st) : run_mx_form<DT, MX_PLAIN, MX_ACT, WM, WN, TM, TN, S>(g, band, most, 0, st);
}

template <int DT>
static int choose_mx_act(const MxGemm& g, bool gated, hipStream_t st) {
    const bool odd = g.N % 8 != 0 || !mx_wide(g.y, g.ldy) || (g.res && !mx_wide(g.res, g.ldr)) || (g.pre && !mx_wide(g.pre, g.ldpre)) || (uintptr_t)g.bias % 16 != 0;
    constexpr long CUS = 256;
    if (((g.a.groups + 7L) / 8) * ((g.w.groups + 7L) / 8) >= 2 * CUS) return run_mx_act<DT, 2, 4, 4, 2, 4>(g, gated, odd, 8, CUS, st);
    return run_mx_act<DT, 2, 2, 2, 2, 4>(g, gated, odd, 8, 2 * CUS, st);
}

int launch_mx_gemm_act(const MxGemm& g, bool gated, hipStream_t st) { return g.dtype == MQ_F16 ? choose_mx_act<MQ_F16>(g, gated, st) : choose_mx_act<MQ_BF16>(g, gated, st); }

}  // namespace mq

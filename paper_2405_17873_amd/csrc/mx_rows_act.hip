// Products of few microscaled rows with an activation or a gate behind them.
#include "mx_rows_core.h"

namespace mq {

// (steps as without an activation)
template <int DT, int KIND>
static int choose_mx_rows_act(const MxRows& r, hipStream_t st) {
    if (r.g.M > 64) return run_mx_rows<DT, true, 4, 4, KIND>(r, st);
    if (r.g.M > 32) return run_mx_rows<DT, true, 2, 2, KIND>(r, st);
    return r.g.w.kq >= 16 ? run_mx_rows<DT, true, 1, 4, KIND>(r, st) : run_mx_rows<DT, true, 1, 2, KIND>(r, st);
}

int launch_mx_rows_act(const MxGemm& g, bool gated, hipStream_t st) {
    MxRows r = {};
    r.g = g;
    if (g.dtype == MQ_F16) return gated ? choose_mx_rows_act<MQ_F16, MX_ACT | MX_GATED>(r, st) : choose_mx_rows_act<MQ_F16, MX_ACT>(r, st);
    return gated ? choose_mx_rows_act<MQ_BF16, MX_ACT | MX_GATED>(r, st) : choose_mx_rows_act<MQ_BF16, MX_ACT>(r, st);
}

}  // namespace mq

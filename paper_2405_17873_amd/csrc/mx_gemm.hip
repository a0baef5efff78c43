// Products of microscaled 4-bit matrices without an activation: which tile.
#include "mx_gemm_core.h"

namespace mq {

template <int DT, int WM, int WN, int TM, int TN, int S>
static int run_mx_gemm(const MxGemm& g, long band, long most, hipStream_t st) {
    if (g.N % 8 != 0 || !mx_wide(g.y, g.ldy) || (g.res && !mx_wide(g.res, g.ldr)) || (uintptr_t)g.bias % 16 != 0)
        return run_mx_form<DT, MX_ODD, 0, 2, 2, 2, 2, 4>(g, band, 1L << 31, 0, st);
    return g.res ? run_mx_form<DT, MX_RES, 0, WM, WN, TM, TN, S>(g, band, most, 0, st) : run_mx_form<DT, MX_PLAIN, 0, WM, WN, TM, TN, S>(g, band, most, 0, st);
}

// Which tile.  A workgroup of 128 x 128 takes 0.48 us for a step of 128 k when it has a compute unit to itself (instructions and latency, not the MFMAs), two
// of them 0.62 us a step between them; one of 256 x 256 takes 1.0 us where the small tiles need 1.24 for as much.  Measured with fp16, M x K x N in us a call
// on activations in MXFP4:
//   256 x 256 from two tiles per compute unit on: 8192 x 8192 x 8192 250 (128 x 128: 309), 7168 x 4096 x 6144 99 (109), 16384 x 1280 x 5120 75 (83),
//   32768 x 320 x 2560 48 (57), with a residual 8192 x 4096 x 4096 91 (101), 16384 x 1280 x 5120 123 (139), 4096 x 1280 x 10240 69 (71).  Without a residual
//   some are no faster, 4096 x 1280 x 10240 44 (44), 17071 x 6144 x 2048 127 (126), 16384 x 640 x 5120 56 (55), and few tiles of five steps slower: 4096 x
//   640 x 10240 32 (29).  With fewer tiles it loses: 16896 x 1536 x 1024 31 (23), 2964 x 1280 x 3840 17.1 (14.2).
//   128 x 160 where that makes one round of what would be one and a part: 4096 x 1280 x 1280 + residual 10.7 (128 x 128: 11.9), 4096 x 5120 x 1280 20.9
//   (23.4), 2461 x 320 x 1920 6.3 (6.8); in other places behind, since its four waves share no weights: 2048 x 2048 x 2048 10.8 (9.3), 2964 x 1280 x 3840 20.2
//   (14.2).
// Several tiles to a workgroup: 16384 x 640 x 5120 54 where one each takes 62, 4096 x 1280 x 10240 43 (48).
template <int DT>
static int choose_mx_gemm(const MxGemm& g, hipStream_t st) {
    auto tiles = [&](long a, long w) { return ((g.a.groups + a - 1) / a) * ((g.w.groups + w - 1) / w); };
    constexpr long CUS = 256;
    if (tiles(8, 8) >= 2 * CUS) return run_mx_gemm<DT, 2, 4, 4, 2, 4>(g, 8, CUS, st);
    if (tiles(4, 4) > CUS && tiles(4, 5) <= CUS) return run_mx_gemm<DT, 4, 1, 1, 5, 6>(g, 8, CUS, st);
    return run_mx_gemm<DT, 2, 2, 2, 2, 4>(g, 8, 2 * CUS, st);
}

int launch_mx_gemm(const MxGemm& g, hipStream_t st) { return g.dtype == MQ_F16 ? choose_mx_gemm<MQ_F16>(g, st) : choose_mx_gemm<MQ_BF16>(g, st); }

}  // namespace mq

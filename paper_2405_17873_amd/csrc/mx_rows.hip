// Products of few rows without an activation: which form.
#include "mx_rows_core.h"

namespace mq {

// us, steps of two 64-k tiles / of a scale word (four tiles): 8 x 1280 x 10240 3.9 / 4.4, 16 x 8192 x 2048 5.7 / 4.9, 8 x 5120 x 20480 (334 MB of
// weights in turn) 16.5 / 15.0, 3.7 TB/s; 48 x 2048 x 640 4.4 / 5.3, 64 x 5120 x 5120 6.9 / 8.2.
template <int DT>
static int choose_mx_rows(const MxRows& r, hipStream_t st) {
    if (r.x) return run_mx_rows<DT, false, 1, 2, 0>(r, st);
    if (r.g.M > 64) return run_mx_rows<DT, true, 4, 4, 0>(r, st);
    if (r.g.M > 32) return run_mx_rows<DT, true, 2, 2, 0>(r, st);
    return r.g.w.kq >= 16 ? run_mx_rows<DT, true, 1, 4, 0>(r, st) : run_mx_rows<DT, true, 1, 2, 0>(r, st);
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

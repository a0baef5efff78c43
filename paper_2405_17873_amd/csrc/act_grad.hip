// Gradient of a linear's activation or gate, and of its bias.
//   y = act(a): da = dy act'(a);  y = v act(g): dv = dy act(g), dg = dy v act'(g);  dbias = sums of da's float32 values over the rows.
// A thread has eight columns of Y and walks down a strip of rows; a workgroup of 32 x 8 threads joins its eight rows' sums in LDS in order, and a second kernel
// those of the strips.  Bound by memory: 2 bytes of dy, of the sums and of da per value.
#include "mx_act.h"

namespace mq {

constexpr int AG_ROWS = 8, AG_COLS = 256;

template <int DT, bool GATED>
__global__ __launch_bounds__(256) void act_grad_kernel(const ActGrad a, int strip) {
    __shared__ float join[AG_ROWS][AG_COLS + 4];
    const int tx = threadIdx.x & 31, ty = threadIdx.x >> 5;
    const int outs = GATED ? a.N >> 1 : a.N, c = (blockIdx.x * 32 + tx) * 8, left = outs - c;
    const long m0 = (long)blockIdx.y * strip, m1 = m0 + strip < a.M ? m0 + strip : a.M;
    float sums[2][8];
#pragma unroll
    for (int e = 0; e < 8; ++e) sums[0][e] = sums[1][e] = 0.0f;
    if (left > 0) {
        for (long m = m0 + ty; m < m1; m += AG_ROWS) {
            const uint4v dv = load8_16(a.dy + m * a.lddy + c, left), av = load8_16(a.pre + m * a.ldpre + c, left);
            uint4v gv = {0, 0, 0, 0};
            if (GATED) gv = load8_16(a.pre + m * a.ldpre + outs + c, left);
            float d0[8], d1[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float dy = T16<DT>::up((uint16_t)(dv[e >> 1] >> (16 * (e & 1)))), v = T16<DT>::up((uint16_t)(av[e >> 1] >> (16 * (e & 1))));
                float slope;
                if (GATED) {
                    const float f = act_and_slope(T16<DT>::up((uint16_t)(gv[e >> 1] >> (16 * (e & 1)))), a.act, slope);
                    d0[e] = dy * f;
                    d1[e] = dy * v * slope;
                    sums[1][e] += d1[e];
                } else {
                    act_and_slope(v, a.act, slope);
                    d0[e] = dy * slope;
                }
                sums[0][e] += d0[e];
            }
            store8_16(a.da + m * a.ldda + c, uint4v{T16<DT>::pack(d0[0], d0[1]), T16<DT>::pack(d0[2], d0[3]), T16<DT>::pack(d0[4], d0[5]), T16<DT>::pack(d0[6], d0[7])}, left);
            if (GATED)
                store8_16(a.da + m * a.ldda + outs + c, uint4v{T16<DT>::pack(d1[0], d1[1]), T16<DT>::pack(d1[2], d1[3]), T16<DT>::pack(d1[4], d1[5]), T16<DT>::pack(d1[6], d1[7])}, left);
        }
    }
    if (!a.dbias) return;
#pragma unroll
    for (int part = 0; part < (GATED ? 2 : 1); ++part) {
        if (part) __syncthreads();
#pragma unroll
        for (int e = 0; e < 8; ++e) join[ty][tx * 8 + e] = sums[part][e];
        __syncthreads();
        const int t = threadIdx.x, col = blockIdx.x * AG_COLS + t;
        if (col < outs) {
            float s = 0.0f;
#pragma unroll
            for (int r = 0; r < AG_ROWS; ++r) s += join[r][t];
            a.partial[(long)blockIdx.y * a.N + part * outs + col] = s;
        }
    }
}

// [strips][N] -> [N]: 64 sums to a workgroup, each in four runs of strips.
__global__ __launch_bounds__(256) void act_grad_join_kernel(const float* partial, int strips, int N, float* dbias) {
    __shared__ float run[4][64];
    const int c = blockIdx.x * 64 + (threadIdx.x & 63), slice = threadIdx.x >> 6;
    float s = 0.0f;
    if (c < N) {
#pragma unroll 8
        for (int p = strips * slice / 4; p < strips * (slice + 1) / 4; ++p) s += partial[(long)p * N + c];
    }
    run[slice][threadIdx.x & 63] = s;
    __syncthreads();
    if (slice == 0 && c < N) dbias[c] = (run[0][c & 63] + run[1][c & 63]) + (run[2][c & 63] + run[3][c & 63]);
}

// Strips of rows: as many as bring the launch to 2048 workgroups, of at least 16 rows.
static int act_grad_strips(long M, long N, bool gated) {
    const long cols = ((gated ? N / 2 : N) + AG_COLS - 1) / AG_COLS;
    long strips = (2048 + cols - 1) / cols;
    if (strips > (M + 15) / 16) strips = (M + 15) / 16;
    return (int)(strips < 1 ? 1 : strips);
}
size_t act_grad_workspace_bytes(long M, long N, bool gated) { return (size_t)act_grad_strips(M, N, gated) * N * 4; }

template <int DT>
static int run_act_grad(const ActGrad& a, hipStream_t st) {
    const int outs = a.gated ? a.N / 2 : a.N;
    int strips = act_grad_strips(a.M, a.N, a.gated);
    const int strip = (int)((a.M + (long)strips - 1) / strips);
    strips = a.M ? (a.M + strip - 1) / strip : 0;
    if (strips > 0) {
        const dim3 grid((unsigned)((outs + AG_COLS - 1) / AG_COLS), (unsigned)strips);
        if (a.gated)
            act_grad_kernel<DT, true><<<grid, 256, 0, st>>>(a, strip);
        else
            act_grad_kernel<DT, false><<<grid, 256, 0, st>>>(a, strip);
        MQ_HIP_CHECK_LAUNCH();
    }
    if (a.dbias) {
        act_grad_join_kernel<<<(unsigned)((a.N + 63) / 64), 256, 0, st>>>(a.partial, strips, a.N, a.dbias);
        MQ_HIP_CHECK_LAUNCH();
    }
    return MQ_OK;
}
int launch_act_grad(const ActGrad& a, hipStream_t st) { return a.dtype == MQ_F16 ? run_act_grad<MQ_F16>(a, st) : run_act_grad<MQ_BF16>(a, st); }

}  // namespace mq

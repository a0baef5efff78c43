// Gradient of a linear's activation or gate, and of its bias.
//   y = act(a): da = dy act'(a);  y = v act(g): dv = dy act(g), dg = dy v act'(g);  dbias = sums of da's float32 values over the rows.
// A thread has eight columns of Y and walks down a strip of rows; a workgroup of 32 x 8 threads joins its eight rows' sums in LDS in order, and a second kernel
// those of the strips.  Bound by memory: 2 bytes of dy, of the sums and of da per value.  4096 x 10240 gated, bfloat16, among others: 41 us (5.1 TB/s), 46 with
// the second kernel; 2964 x 1280 5.2 and 9.0.  Earlier, on another card, 38.5 with the second kernel, 58 with loads in branches and none ahead, and with 512 / 1024 / 2048 / 4096
// workgroups in all 40.8 / 39.5 / 38.5 / 41.5.
#include "mx_act.h"

namespace mq {

constexpr int AG_ROWS = 8, AG_COLS = 256;

// Eight gradients da (gated: and the gates'), added to the sums.
template <int DT, bool GATED>
__device__ __forceinline__ void act_grad_values(uint4v dv, uint4v av, uint4v gv, int act, float (*sums)[8], uint4v* out) {
    float d[2][8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const float dy = T16<DT>::up((uint16_t)(dv[e >> 1] >> (16 * (e & 1)))), v = T16<DT>::up((uint16_t)(av[e >> 1] >> (16 * (e & 1))));
        float slope;
        if (GATED) {
            const float f = act_and_slope(T16<DT>::up((uint16_t)(gv[e >> 1] >> (16 * (e & 1)))), act, slope);
            d[0][e] = dy * f;
            d[1][e] = dy * v * slope;
            sums[1][e] += d[1][e];
        } else {
            act_and_slope(v, act, slope);
            d[0][e] = dy * slope;
        }
        sums[0][e] += d[0][e];
    }
#pragma unroll
    for (int p = 0; p < (GATED ? 2 : 1); ++p)
        out[p] = uint4v{T16<DT>::pack(d[p][0], d[p][1]), T16<DT>::pack(d[p][2], d[p][3]), T16<DT>::pack(d[p][4], d[p][5]), T16<DT>::pack(d[p][6], d[p][7])};
}

// ACT: the activation.  WIDE: rows on 16-byte boundaries, whole vectors of eight; the loads of the next row are then under way while one is computed.
template <int DT, bool GATED, int ACT, bool WIDE>
__global__ __launch_bounds__(256) void act_grad_kernel(const ActGrad a, int strip) {
    __shared__ float join[AG_ROWS][AG_COLS + 4];
    const int tx = threadIdx.x & 31, ty = threadIdx.x >> 5;
    const int outs = GATED ? a.N >> 1 : a.N, c = (blockIdx.x * 32 + tx) * 8, left = outs - c;
    const long m0 = (long)blockIdx.y * strip, m1 = m0 + strip < a.M ? m0 + strip : a.M;
    float sums[2][8];
#pragma unroll
    for (int e = 0; e < 8; ++e) sums[0][e] = sums[1][e] = 0.0f;
    if (left > 0 && m0 + ty < m1) {
        auto load = [&](const uint16_t* p) { return WIDE ? *(const uint4v*)p : load8_16(p, left); };
        auto store = [&](uint16_t* p, uint4v v) {
            if (WIDE)
                __builtin_nontemporal_store(v, (uint4v*)p);
            else
                store8_16(p, v, left);
        };
        const uint16_t *dy = a.dy + c, *pre = a.pre + c;
        long m = m0 + ty;
        uint4v d = load(dy + m * a.lddy), v = load(pre + m * a.ldpre), g = {0, 0, 0, 0};
        if (GATED) g = load(pre + m * a.ldpre + outs);
        while (true) {
            // (the last row's loads are its own once more: no branch)
            const long next = m + AG_ROWS < m1 ? m + AG_ROWS : m;
            const uint4v d1 = load(dy + next * a.lddy), v1 = load(pre + next * a.ldpre), g1 = GATED ? load(pre + next * a.ldpre + outs) : uint4v{0, 0, 0, 0};
            uint4v out[2];
            act_grad_values<DT, GATED>(d, v, g, ACT, sums, out);
            store(a.da + m * a.ldda + c, out[0]);
            if (GATED) store(a.da + m * a.ldda + outs + c, out[1]);
            if (m + AG_ROWS >= m1) break;
            m = next, d = d1, v = v1, g = g1;
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

// [strips][N] -> [N]: eight sums to a workgroup, each in 32 runs of strips.
__global__ __launch_bounds__(256) void act_grad_join_kernel(const float* partial, int strips, int N, float* dbias) {
    __shared__ float run[32][8];
    const int e = threadIdx.x & 7, c = blockIdx.x * 8 + e, slice = threadIdx.x >> 3;
    float s = 0.0f;
    if (c < N) {
#pragma unroll 4
        for (int p = slice; p < strips; p += 32) s += partial[(long)p * N + c];
    }
    run[slice][e] = s;
    __syncthreads();
    if (slice == 0 && c < N) {
        s = 0.0f;
        for (int i = 0; i < 32; ++i) s += run[i][e];
        dbias[c] = s;
    }
}

// Strips of rows: as many as bring the launch to 2048 workgroups, of at least 16 rows.
static int act_grad_strips(long M, long N, bool gated) {
    const long cols = ((gated ? N / 2 : N) + AG_COLS - 1) / AG_COLS;
    long strips = (2048 + cols - 1) / cols;
    if (strips > (M + 15) / 16) strips = (M + 15) / 16;
    return (int)(strips < 1 ? 1 : strips);
}
size_t act_grad_workspace_bytes(long M, long N, bool gated) { return (size_t)act_grad_strips(M, N, gated) * N * 4; }

template <int DT, bool GATED, int ACT>
static void start_act_grad(const ActGrad& a, dim3 grid, int strip, hipStream_t st) {
    auto wide = [&](const void* p, long ld) { return (uintptr_t)p % 16 == 0 && (a.M == 1 || ld % 8 == 0); };
    if ((GATED ? a.N / 2 : a.N) % 8 == 0 && wide(a.dy, a.lddy) && wide(a.pre, a.ldpre) && wide(a.da, a.ldda))
        act_grad_kernel<DT, GATED, ACT, true><<<grid, 256, 0, st>>>(a, strip);
    else
        act_grad_kernel<DT, GATED, ACT, false><<<grid, 256, 0, st>>>(a, strip);
}
template <int DT, bool GATED>
static int run_act_grad(const ActGrad& a, hipStream_t st) {
    const int outs = GATED ? a.N / 2 : a.N;
    int strips = act_grad_strips(a.M, a.N, GATED);
    const int strip = (int)((a.M + (long)strips - 1) / strips);
    strips = a.M ? (a.M + strip - 1) / strip : 0;
    if (strips > 0) {
        const dim3 grid((unsigned)((outs + AG_COLS - 1) / AG_COLS), (unsigned)strips);
        if (a.act == MQ_ACT_GELU)
            start_act_grad<DT, GATED, MQ_ACT_GELU>(a, grid, strip, st);
        else if (a.act == MQ_ACT_SILU)
            start_act_grad<DT, GATED, MQ_ACT_SILU>(a, grid, strip, st);
        else
            start_act_grad<DT, GATED, MQ_ACT_GELU_TANH>(a, grid, strip, st);
        MQ_HIP_CHECK_LAUNCH();
    }
    if (a.dbias) {
        act_grad_join_kernel<<<(unsigned)((a.N + 7) / 8), 256, 0, st>>>(a.partial, strips, a.N, a.dbias);
        MQ_HIP_CHECK_LAUNCH();
    }
    return MQ_OK;
}
int launch_act_grad(const ActGrad& a, hipStream_t st) {
    if (a.dtype == MQ_F16) return a.gated ? run_act_grad<MQ_F16, true>(a, st) : run_act_grad<MQ_F16, false>(a, st);
    return a.gated ? run_act_grad<MQ_BF16, true>(a, st) : run_act_grad<MQ_BF16, false>(a, st);
}

}  // namespace mq

// Norm of every query and key head and its rotation by position, in one pass, and the gradient of both.
//
// A head is held by L lanes with NU units of eight values each (L NU of them, D / 8 used): a unit is four pairs, whose values lie together (interleaved) or
// R / 2 apart, or, past the R values that turn, eight values.  Both values of a pair are in one lane, and a lane's pairs are the same in every head
// of a row, so that an angle's sine and cosine are computed once for the heads that a wave takes of a row.
//   y = T(x r w), r = 1 / sqrt(mean x^2 + eps), T the rotation of pair p by angle position[axis p] f_p
//   g = T^-1 dy, dw = sum g x r, dx = r (g w - x r^2 mean(g w x))
// Angles: f / (2 pi) is a 64-bit fraction of a turn; its product with a position, modulo one turn, is exact integer arithmetic however far the position is.
#include "lane_sum.h"
#include "mx_common.h"

namespace mq {

typedef uint2v uint2v_half __attribute__((aligned(2)));

struct HeadUnit {
    float re[4], im[4];
};

// Sine and cosine of a 32-bit fraction of a turn: a quarter turn around zero is left after the quadrant, and the Taylor series to x^9 and x^8 are good to
// 2 10^-9 and 3 10^-8 there.
__device__ __forceinline__ void turn_sincos(uint32_t t, float& s, float& c) {
    const uint32_t q = (t + 0x20000000u) >> 30;
    const float x = (float)(int32_t)(t - (q << 30)) * 1.4629180792671596e-9f, z = x * x;  // 2 pi / 2^32
    const float ps = x + x * z * (-1.6666667e-1f + z * (8.3333333e-3f + z * (-1.9841270e-4f + z * 2.7557319e-6f)));
    const float pc = 1.0f + z * (-0.5f + z * (4.1666668e-2f + z * (-1.3888889e-3f + z * 2.4801587e-5f)));
    s = q & 1 ? pc : ps;
    c = q & 1 ? ps : pc;
    if (q & 2) s = -s;
    if ((q + 1) & 2) c = -c;
}

__device__ __forceinline__ float head_param(const void* p, int dtype, int i) {
    if (dtype == MQ_F32) return ((const float*)p)[i];
    const uint16_t b = ((const uint16_t*)p)[i];
    return dtype == MQ_F16 ? T16<MQ_F16>::up(b) : T16<MQ_BF16>::up(b);
}

// What a lane knows of its units: where their two runs of four values start in a head, whether they exist, and whether they turn.
template <int L, int NU>
struct HeadLane {
    int lo[NU], hi[NU], first[NU];
    bool in[NU], turns[NU];
    __device__ __forceinline__ HeadLane(const HeadArgs& a, int sub, bool interleaved) {
#pragma unroll
        for (int i = 0; i < NU; ++i) {
            const int u = i * L + sub;
            in[i] = u * 8 < a.D;
            turns[i] = u * 4 < a.pairs;
            first[i] = u * 4;
            const bool split = turns[i] && !interleaved;
            lo[i] = in[i] ? (split ? u * 4 : u * 8) : 0;
            hi[i] = in[i] ? (split ? a.pairs + u * 4 : u * 8 + 4) : 4;
        }
    }
};

template <int L, int NU>
__device__ __forceinline__ void head_angles(const HeadArgs& a, const HeadLane<L, NU>& lane, long row, float (*sn)[4], float (*cs)[4]) {
    uint2v pos[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        pos[i] = uint2v{0, 0};
        if (i < a.axes) {
            const long at = row * a.ldpos + i;
            if (a.pos_bytes == 8) {
                const unsigned long long v = ((const unsigned long long*)a.pos)[at];
                pos[i] = uint2v{(uint32_t)v, (uint32_t)(v >> 32)};
            } else {
                const int v = ((const int*)a.pos)[at];
                pos[i] = uint2v{(uint32_t)v, (uint32_t)(v >> 31)};
            }
        }
    }
#pragma unroll
    for (int i = 0; i < NU; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            sn[i][j] = 0.0f, cs[i][j] = 1.0f;
            if (lane.turns[i]) {
                const uint4v f = a.table[lane.first[i] + j];  // a turn's fraction (low, high), axis
                uint32_t p0 = pos[0][0], p1 = pos[0][1];
#pragma unroll
                for (int k = 1; k < 4; ++k) p0 = f[2] == (uint32_t)k ? pos[k][0] : p0, p1 = f[2] == (uint32_t)k ? pos[k][1] : p1;
                turn_sincos(f[1] * p0 + __umulhi(f[0], p0) + f[0] * p1, sn[i][j], cs[i][j]);
            }
        }
}

// Four raw pairs of a unit into numbers.
template <int DT, bool INTER>
__device__ __forceinline__ HeadUnit head_widen(uint2v lo, uint2v hi) {
    HeadUnit u;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const float a = T16<DT>::up((uint16_t)(lo[j >> 1] >> (16 * (j & 1)))), b = T16<DT>::up((uint16_t)(hi[j >> 1] >> (16 * (j & 1))));
        if (!INTER) {
            u.re[j] = a, u.im[j] = b;
        } else if (j & 1) {
            u.im[j >> 1] = a, u.im[2 + (j >> 1)] = b;
        } else {
            u.re[j >> 1] = a, u.re[2 + (j >> 1)] = b;
        }
    }
    return u;
}
template <int DT, bool INTER>
__device__ __forceinline__ void head_pack(const HeadUnit& u, uint2v& lo, uint2v& hi) {
    if (INTER) {
        lo = uint2v{T16<DT>::pack(u.re[0], u.im[0]), T16<DT>::pack(u.re[1], u.im[1])};
        hi = uint2v{T16<DT>::pack(u.re[2], u.im[2]), T16<DT>::pack(u.re[3], u.im[3])};
    } else {
        lo = uint2v{T16<DT>::pack(u.re[0], u.re[1]), T16<DT>::pack(u.re[2], u.re[3])};
        hi = uint2v{T16<DT>::pack(u.im[0], u.im[1]), T16<DT>::pack(u.im[2], u.im[3])};
    }
}
template <bool INTER>
__device__ __forceinline__ int head_value(int j, bool im) {  // which of a unit's eight values (0 .. 3 the first run) pair j's is
    return INTER ? 2 * j + im : 4 * im + j;
}

template <int DT, int L, int NU, bool INTER>
__device__ __forceinline__ void head_weights(const HeadArgs& a, const HeadLane<L, NU>& lane, const void* p, HeadUnit* w) {
#pragma unroll
    for (int i = 0; i < NU; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int r = head_value<INTER>(j, false), m = head_value<INTER>(j, true);
            w[i].re[j] = p && lane.in[i] ? head_param(p, a.param_dtype, (r < 4 ? lane.lo[i] : lane.hi[i] - 4) + r) : 1.0f;
            w[i].im[j] = p && lane.in[i] ? head_param(p, a.param_dtype, (m < 4 ? lane.lo[i] : lane.hi[i] - 4) + m) : 1.0f;
        }
}
__device__ __forceinline__ HeadUnit head_either(bool first, const HeadUnit& a, const HeadUnit& b) {
    HeadUnit u;
#pragma unroll
    for (int j = 0; j < 4; ++j) u.re[j] = first ? a.re[j] : b.re[j], u.im[j] = first ? a.im[j] : b.im[j];
    return u;
}
// (What does not turn stays as it is, infinities included.)
__device__ __forceinline__ HeadUnit head_turn(const HeadUnit& u, const float* s, const float* c, bool turns, float way) {
    HeadUnit o;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const float sj = s[j] * way;
        o.re[j] = turns ? u.re[j] * c[j] - u.im[j] * sj : u.re[j];
        o.im[j] = turns ? u.re[j] * sj + u.im[j] * c[j] : u.im[j];
    }
    return o;
}

// A wave takes a chunk of the heads of one row, 64 / L of them at a time and U such turns in flight.
template <int DT, int L, int NU, bool INTER>
__global__ __launch_bounds__(256) void heads_kernel(const HeadArgs a) {
    constexpr int G = 64 / L, U = NU == 1 ? 4 : NU == 3 ? 2 : 1;
    const int ln = threadIdx.x & 63, grp = ln / L;
    const uint32_t task = __builtin_amdgcn_readfirstlane(blockIdx.x * 4 + (threadIdx.x >> 6));
    uint32_t row_v, chunk_v;
    a.chunks.divmod(task, row_v, chunk_v);
    const int row = __builtin_amdgcn_readfirstlane((int)row_v), chunk = __builtin_amdgcn_readfirstlane((int)chunk_v);
    if (row >= a.M) return;
    const int H = a.q + a.k, h0 = chunk * a.per_chunk, h1 = h0 + a.per_chunk < H ? h0 + a.per_chunk : H;
    const HeadLane<L, NU> lane(a, ln % L, INTER);
    const uint16_t* x = a.x + row * a.ldx;
    uint16_t* y = a.y + row * a.ldy;
    float sn[NU][4], cs[NU][4];
    HeadUnit wq[NU], wk[NU];
    const float mean = 1.0f / (float)a.D;
    for (int base = h0; base < h1; base += G * U) {
        uint2v lo[U][NU], hi[U][NU];
#pragma unroll
        for (int t = 0; t < U; ++t) {
            const int h = base + t * G + grp;
#pragma unroll
            for (int i = 0; i < NU; ++i) {
                const bool in = h < h1 && lane.in[i];
                const uint16_t* p = x + (in ? h * a.D : 0);
                lo[t][i] = in ? *(const uint2v_half*)(p + lane.lo[i]) : uint2v{0, 0};
                hi[t][i] = in ? *(const uint2v_half*)(p + lane.hi[i]) : uint2v{0, 0};
            }
        }
        if (base == h0) {
            head_angles<L, NU>(a, lane, row, sn, cs);
            head_weights<DT, L, NU, INTER>(a, lane, a.qw, wq);
            head_weights<DT, L, NU, INTER>(a, lane, a.kw, wk);
        }
#pragma unroll
        for (int t = 0; t < U; ++t) {
            const int h = base + t * G + grp;
            HeadUnit u[NU];
            float sum = 0.0f;
#pragma unroll
            for (int i = 0; i < NU; ++i) {
                u[i] = head_widen<DT, INTER>(lo[t][i], hi[t][i]);
#pragma unroll
                for (int j = 0; j < 4; ++j) sum += u[i].re[j] * u[i].re[j] + u[i].im[j] * u[i].im[j];
            }
            if (a.norm) {
                const float r = rsqrtf(lane_sum<L>(sum) * mean + a.eps);
#pragma unroll
                for (int i = 0; i < NU; ++i) {
                    const HeadUnit w = head_either(h < a.q, wq[i], wk[i]);
#pragma unroll
                    for (int j = 0; j < 4; ++j) u[i].re[j] = u[i].re[j] * r * w.re[j], u[i].im[j] = u[i].im[j] * r * w.im[j];
                }
            }
#pragma unroll
            for (int i = 0; i < NU; ++i) {
                uint2v o0, o1;
                head_pack<DT, INTER>(head_turn(u[i], sn[i], cs[i], lane.turns[i], 1.0f), o0, o1);
                if (h < h1 && lane.in[i]) {
                    *(uint2v_half*)(y + h * a.D + lane.lo[i]) = o0;
                    *(uint2v_half*)(y + h * a.D + lane.hi[i]) = o1;
                }
            }
        }
    }
}

// The gradient: waves walk over the rows (and chunks of their heads), and hold the sums for the weights of their units; a workgroup joins those of its
// lanes and waves in a fixed order, and a second kernel those of the workgroups.
template <int DT, int L, int NU, bool INTER>
__global__ __launch_bounds__(256) void heads_grad_kernel(const HeadArgs a) {
    constexpr int G = 64 / L, U = NU == 1 ? 2 : 1;
    __shared__ float join[4 * 64 * NU * 8];
    const int ln = threadIdx.x & 63, wv = threadIdx.x >> 6, grp = ln / L, sub = ln % L;
    const HeadLane<L, NU> lane(a, sub, INTER);
    HeadUnit wq[NU], wk[NU], sums[2][NU];
    head_weights<DT, L, NU, INTER>(a, lane, a.qw, wq);
    head_weights<DT, L, NU, INTER>(a, lane, a.kw, wk);
#pragma unroll
    for (int i = 0; i < NU; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) sums[0][i].re[j] = sums[0][i].im[j] = sums[1][i].re[j] = sums[1][i].im[j] = 0.0f;
    const int H = a.q + a.k;
    const float mean = 1.0f / (float)a.D;
    for (uint32_t task_v = blockIdx.x * 4 + wv; task_v < a.tasks; task_v += gridDim.x * 4) {
        const uint32_t task = __builtin_amdgcn_readfirstlane(task_v);
        uint32_t row_v, chunk_v;
        a.chunks.divmod(task, row_v, chunk_v);
        const int row = __builtin_amdgcn_readfirstlane((int)row_v), chunk = __builtin_amdgcn_readfirstlane((int)chunk_v);
        const int h0 = chunk * a.per_chunk, h1 = h0 + a.per_chunk < H ? h0 + a.per_chunk : H;
        const uint16_t *x = a.x + row * a.ldx, *dy = a.dy + row * a.lddy;
        uint16_t* dx = a.dx + row * a.lddx;
        float sn[NU][4], cs[NU][4];
        for (int base = h0; base < h1; base += G * U) {
            uint2v lo[U][NU], hi[U][NU], dlo[U][NU], dhi[U][NU];
#pragma unroll
            for (int t = 0; t < U; ++t) {
                const int h = base + t * G + grp;
#pragma unroll
                for (int i = 0; i < NU; ++i) {
                    const bool in = h < h1 && lane.in[i];
                    const int at = in ? h * a.D : 0;
                    dlo[t][i] = in ? *(const uint2v_half*)(dy + at + lane.lo[i]) : uint2v{0, 0};
                    dhi[t][i] = in ? *(const uint2v_half*)(dy + at + lane.hi[i]) : uint2v{0, 0};
                    lo[t][i] = in && a.norm ? *(const uint2v_half*)(x + at + lane.lo[i]) : uint2v{0, 0};
                    hi[t][i] = in && a.norm ? *(const uint2v_half*)(x + at + lane.hi[i]) : uint2v{0, 0};
                }
            }
            if (base == h0) head_angles<L, NU>(a, lane, row, sn, cs);
#pragma unroll
            for (int t = 0; t < U; ++t) {
                const int h = base + t * G + grp;
                const bool is_q = h < a.q, live = h < h1;
                HeadUnit g[NU];
#pragma unroll
                for (int i = 0; i < NU; ++i) g[i] = head_turn(head_widen<DT, INTER>(dlo[t][i], dhi[t][i]), sn[i], cs[i], lane.turns[i], -1.0f);
                if (a.norm) {
                    HeadUnit v[NU];
                    float sq = 0.0f, dot = 0.0f;
#pragma unroll
                    for (int i = 0; i < NU; ++i) {
                        v[i] = head_widen<DT, INTER>(lo[t][i], hi[t][i]);
                        const HeadUnit w = head_either(is_q, wq[i], wk[i]);
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            sq += v[i].re[j] * v[i].re[j] + v[i].im[j] * v[i].im[j];
                            dot += g[i].re[j] * w.re[j] * v[i].re[j] + g[i].im[j] * w.im[j] * v[i].im[j];
                        }
                    }
                    const float r = rsqrtf(lane_sum<L>(sq) * mean + a.eps), back = lane_sum<L>(dot) * mean * r * r;
#pragma unroll
                    for (int i = 0; i < NU; ++i) {
                        const HeadUnit w = head_either(is_q, wq[i], wk[i]);
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            const float dr = live ? g[i].re[j] * (v[i].re[j] * r) : 0.0f, di = live ? g[i].im[j] * (v[i].im[j] * r) : 0.0f;
                            sums[0][i].re[j] += is_q ? dr : 0.0f, sums[0][i].im[j] += is_q ? di : 0.0f;
                            sums[1][i].re[j] += is_q ? 0.0f : dr, sums[1][i].im[j] += is_q ? 0.0f : di;
                            g[i].re[j] = r * (g[i].re[j] * w.re[j] - v[i].re[j] * back);
                            g[i].im[j] = r * (g[i].im[j] * w.im[j] - v[i].im[j] * back);
                        }
                    }
                }
#pragma unroll
                for (int i = 0; i < NU; ++i) {
                    uint2v o0, o1;
                    head_pack<DT, INTER>(g[i], o0, o1);
                    if (live && lane.in[i]) {
                        *(uint2v_half*)(dx + h * a.D + lane.lo[i]) = o0;
                        *(uint2v_half*)(dx + h * a.D + lane.hi[i]) = o1;
                    }
                }
            }
        }
    }
    if (!a.partial) return;
#pragma unroll
    for (int part = 0; part < 2; ++part) {
        if (part) __syncthreads();
#pragma unroll
        for (int i = 0; i < NU; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                float* p = join + (wv * G + grp) * (L * NU * 8) + (i * L + sub) * 8;
                p[head_value<INTER>(j, false)] = sums[part][i].re[j];
                p[head_value<INTER>(j, true)] = sums[part][i].im[j];
            }
        __syncthreads();
        for (int c = threadIdx.x; c < a.D; c += 256) {
            float s = 0.0f;
            for (int w = 0; w < 4 * G; ++w) s += join[w * (L * NU * 8) + c];
            const int u = c >> 3, e = c & 7;
            const int at = u * 4 < a.pairs && !INTER ? (e < 4 ? u * 4 + e : a.pairs + u * 4 + e - 4) : c;
            a.partial[((long)blockIdx.x * 2 + part) * a.D + at] = s;
        }
    }
}

// [parts][2 D] -> two vectors of D: 64 sums to a workgroup, each in four runs of parts.
__global__ __launch_bounds__(256) void heads_join_kernel(const float* partial, int parts, int D, float* dq, float* dk) {
    __shared__ float run[4][64];
    const int c = blockIdx.x * 64 + (threadIdx.x & 63), slice = threadIdx.x >> 6;
    float s = 0.0f;
    if (c < 2 * D) {
#pragma unroll 8
        for (int p = parts * slice / 4; p < parts * (slice + 1) / 4; ++p) s += partial[(long)p * 2 * D + c];
    }
    run[slice][threadIdx.x & 63] = s;
    __syncthreads();
    if (slice == 0 && c < 2 * D) {
        s = (run[0][c & 63] + run[1][c & 63]) + (run[2][c & 63] + run[3][c & 63]);
        float* out = c < D ? dq : dk;
        if (out) out[c < D ? c : c - D] = s;
    }
}

// Workgroups of the gradient, and so parts of its sums: at most as many as the chip holds at once.
static long heads_grad_workgroups(long tasks) { return tasks <= 0 ? 0 : (tasks + 3) / 4 < 1024 ? (tasks + 3) / 4 : 1024; }
// Waves for every row: as many as bring the launch to 2048 (eight per compute unit), but no part of a turn's heads.
static void heads_chunks(HeadArgs& a, int L) {
    const int H = a.q + a.k, G = 64 / L, turns = (H + G - 1) / G;
    long want = a.M > 0 ? (2048 + a.M - 1) / a.M : 1;
    if (want > turns) want = turns;
    const int per = (int)((turns + want - 1) / want);
    a.per_chunk = per * G;
    const int chunks = (turns + per - 1) / per;
    a.chunks = FastDiv::make((uint32_t)chunks);
    a.tasks = (uint32_t)((long)a.M * chunks);
}

template <int DT, int L, int NU>
static int run_heads(HeadArgs& a, bool grad, hipStream_t st) {
    heads_chunks(a, L);
    if (!grad) {
        const unsigned wgs = (unsigned)(((long)a.tasks + 3) / 4);
        if (a.interleaved)
            heads_kernel<DT, L, NU, true><<<wgs, 256, 0, st>>>(a);
        else
            heads_kernel<DT, L, NU, false><<<wgs, 256, 0, st>>>(a);
        MQ_HIP_CHECK_LAUNCH();
        return MQ_OK;
    }
    const long wgs = heads_grad_workgroups(a.tasks);
    if (!a.dq_weight && !a.dk_weight) a.partial = nullptr;
    if (wgs > 0) {
        if (a.interleaved)
            heads_grad_kernel<DT, L, NU, true><<<(unsigned)wgs, 256, 0, st>>>(a);
        else
            heads_grad_kernel<DT, L, NU, false><<<(unsigned)wgs, 256, 0, st>>>(a);
        MQ_HIP_CHECK_LAUNCH();
    }
    if (a.dq_weight || a.dk_weight) {
        heads_join_kernel<<<(unsigned)((2 * a.D + 63) / 64), 256, 0, st>>>(a.partial, (int)wgs, a.D, a.dq_weight, a.dk_weight);
        MQ_HIP_CHECK_LAUNCH();
    }
    return MQ_OK;
}
// Lanes and units for a head of n units of eight values: the fewest idle ones.
template <int DT>
static int choose_heads(HeadArgs& a, bool grad, hipStream_t st) {
    const int n = a.D / 8;
    if (n <= 1) return run_heads<DT, 1, 1>(a, grad, st);
    if (n <= 2) return run_heads<DT, 2, 1>(a, grad, st);
    if (n <= 3) return run_heads<DT, 1, 3>(a, grad, st);
    if (n <= 4) return run_heads<DT, 4, 1>(a, grad, st);
    if (n <= 5) return run_heads<DT, 1, 5>(a, grad, st);
    if (n <= 6) return run_heads<DT, 2, 3>(a, grad, st);
    if (n <= 8) return run_heads<DT, 8, 1>(a, grad, st);
    if (n <= 10) return run_heads<DT, 2, 5>(a, grad, st);
    if (n <= 12) return run_heads<DT, 4, 3>(a, grad, st);
    if (n <= 16) return run_heads<DT, 16, 1>(a, grad, st);
    if (n <= 20) return run_heads<DT, 4, 5>(a, grad, st);
    if (n <= 24) return run_heads<DT, 8, 3>(a, grad, st);
    if (n <= 32) return run_heads<DT, 32, 1>(a, grad, st);
    return run_heads<DT, 64, 1>(a, grad, st);
}

size_t heads_grad_workspace_bytes(long M, int H, int D) {
    // (a wave takes at least one head)
    return (size_t)heads_grad_workgroups(M * H) * 2 * D * 4;
}
int launch_heads(HeadArgs& a, bool grad, hipStream_t st) { return a.dtype == MQ_F16 ? choose_heads<MQ_F16>(a, grad, st) : choose_heads<MQ_BF16>(a, grad, st); }

}  // namespace mq

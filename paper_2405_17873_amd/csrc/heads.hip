// Norm of every query and key head and its rotation by position, in one pass, and the gradient of both.
//
// A head is held by L lanes (a power of two; D / 8 of them used) with a unit of eight values each: four pairs, whose values lie together (interleaved) or R / 2
// apart, or, past the R values that turn, eight values.  Both values of a pair are in one lane, and a lane's pairs are the same in every head of a row, so that an
// angle's sine and cosine are computed once for the heads that a wave takes of a row.  Waves walk over the rows; what depends on the lane alone stays in registers.
//   y = T(x r w), r = 1 / sqrt(mean x^2 + eps), T the rotation of pair p by angle position[axis p] f_p
//   g = T^-1 dy, dw = sum g x r, dx = r (g w - x r mean(g w x r))
// Bound by memory.  us a call among others (bfloat16): forward 32768 x 40 heads of 64, three axes 62 (5.4 TB/s), 4096 x 40 of 128 14.6, gradient 103 and 27 to 30, 4 of it joining
// the sums; 64-bit positions the same; the rotation alone 60 and 13.8.  (Lanes with three or five units each, so that none is idle with heads of 96 or 80, needed 200
// registers and more: 2964 x 32 heads of 80 50; sine and cosine as polynomials, weights and table once per row 90 where the first takes 63.)
// Angles: f / (2 pi) is a 64-bit fraction of a turn; its product with a position, modulo one turn, is exact integer arithmetic however far the position is.
#include "lane_sum.h"
#include "mx_common.h"

namespace mq {

typedef uint2v uint2v_half __attribute__((aligned(2)));

struct HeadUnit {  // (vectors: arrays of floats that are read in other pairs than they were written in went through LDS, 8 -> 20 us of 2964 x 32 heads of 80)
    float4v re, im;
};

// A row's positions: lane k has that of axis k modulo 4 (or the last).  (Scalar loads would be waited for one by one, some 0.5 us each.)
struct HeadPosition {
    uint32_t low, high;
    __device__ __forceinline__ void load(const HeadArgs& a, long row) {
        const __amdgpu_buffer_rsrc_t r = __builtin_amdgcn_make_buffer_rsrc((void*)((const char*)a.pos + row * a.ldpos * a.pos_bytes), 0, a.axes * a.pos_bytes, 0x00020000);
        const int k = threadIdx.x & 3, at = (k < a.axes ? k : a.axes - 1) * a.pos_bytes;
        low = (uint32_t)__builtin_amdgcn_raw_buffer_load_b32(r, at, 0, 0);
        high = (uint32_t)__builtin_amdgcn_raw_buffer_load_b32(r, at + a.pos_bytes - 4, 0, 0);
    }
};
// Where a wave is in its tasks: chunks of the heads of a row, `step` heads at a time.
struct HeadWalk {
    uint32_t task;
    int row, base, end;
    __device__ __forceinline__ void enter(const HeadArgs& a) {
        uint32_t row_v, chunk_v;
        a.chunks.divmod(task, row_v, chunk_v);
        const int chunk = __builtin_amdgcn_readfirstlane((int)chunk_v), H = a.q + a.k;
        row = __builtin_amdgcn_readfirstlane((int)row_v);
        base = chunk * a.per_chunk;
        end = base + a.per_chunk < H ? base + a.per_chunk : H;
    }
    __device__ __forceinline__ HeadWalk(const HeadArgs& a, uint32_t first) : task(__builtin_amdgcn_readfirstlane(first)), row(0), base(0), end(0) {
        if (more(a)) enter(a);
    }
    __device__ __forceinline__ bool more(const HeadArgs& a) const { return task < a.tasks; }
    __device__ __forceinline__ void next(const HeadArgs& a, int step, uint32_t waves) {
        base += step;
        if (base < end) return;
        task += waves;
        if (more(a)) enter(a);
    }
};

// What a lane knows of its unit: where its two runs of four values start in a head, whether it exists, and whether it turns; its pairs' fractions and axes.
template <int L, bool INTER>
struct HeadLane {
    int first, lo, hi;
    bool in, turns;
    uint4v f0, f1, axis;
    __device__ __forceinline__ HeadLane(const HeadArgs& a, int sub) {
        first = sub * 4;
        in = sub * 8 < a.D;
        turns = sub * 4 < a.pairs;
        const bool split = turns && !INTER;
        lo = in ? (split ? sub * 4 : sub * 8) : 0;
        hi = in ? (split ? a.pairs + sub * 4 : sub * 8 + 4) : 4;
    }
    __device__ __forceinline__ void load_table(const HeadArgs& a) {  // (zeros where nothing turns)
        const __amdgpu_buffer_rsrc_t r = __builtin_amdgcn_make_buffer_rsrc((void*)a.table, 0, a.pairs * 16, 0x00020000);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const uint4v f = __builtin_amdgcn_raw_buffer_load_b128(r, (first + j) * 16, 0, 0);  // a turn's fraction (low, high), axis
            f0[j] = f[0], f1[j] = f[1], axis[j] = f[2];
        }
    }
    // Sines and cosines of a row: those of a lane that does not turn are 0 and 1.  The hardware's functions take turns (measured: off by at most
    // 2 10^-7 over a turn).
    __device__ __forceinline__ void angles(const HeadArgs& a, const HeadPosition& p, float4v& s, float4v& c) const {
        if (a.axes == 0) {
#pragma unroll
            for (int j = 0; j < 4; ++j) s[j] = 0.0f, c[j] = 1.0f;
            return;
        }
        uint4v t, p0, p1;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            p0[k] = (uint32_t)__builtin_amdgcn_readlane((int)p.low, k);
            p1[k] = a.pos_bytes == 8 ? (uint32_t)__builtin_amdgcn_readlane((int)p.high, k) : (uint32_t)((int)p0[k] >> 31);
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            uint32_t q0 = p0[0], q1 = p1[0];
            if (a.axes > 1) {
#pragma unroll
                for (int k = 1; k < 4; ++k) q0 = axis[j] == (uint32_t)k ? p0[k] : q0, q1 = axis[j] == (uint32_t)k ? p1[k] : q1;
            }
            t[j] = f1[j] * q0 + __umulhi(f0[j], q0);
            t[j] += a.pos_bytes == 8 ? f0[j] * q1 : q1 ? 0u - f0[j] : 0u;
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const float turn = (float)(int32_t)t[j] * 2.3283064e-10f;  // 2^-32
            s[j] = __builtin_amdgcn_sinf(turn);
            c[j] = __builtin_amdgcn_cosf(turn);
        }
    }
    // Four raw pairs into numbers, and back.
    template <int DT>
    static __device__ __forceinline__ HeadUnit widen(uint4v v) {
        HeadUnit u;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int r = INTER ? 2 * j : j, m = INTER ? 2 * j + 1 : 4 + j;
            u.re[j] = T16<DT>::up((uint16_t)(v[r >> 1] >> (16 * (r & 1))));
            u.im[j] = T16<DT>::up((uint16_t)(v[m >> 1] >> (16 * (m & 1))));
        }
        return u;
    }
    template <int DT>
    static __device__ __forceinline__ uint4v pack(const HeadUnit& u) {
        if (INTER)
            return uint4v{T16<DT>::pack(u.re[0], u.im[0]), T16<DT>::pack(u.re[1], u.im[1]), T16<DT>::pack(u.re[2], u.im[2]), T16<DT>::pack(u.re[3], u.im[3])};
        return uint4v{T16<DT>::pack(u.re[0], u.re[1]), T16<DT>::pack(u.re[2], u.re[3]), T16<DT>::pack(u.im[0], u.im[1]), T16<DT>::pack(u.im[2], u.im[3])};
    }
    __device__ __forceinline__ uint4v load(const uint16_t* head) const {
        if (INTER) return *(const uint4v_any*)(head + lo);
        const uint2v a = *(const uint2v_half*)(head + lo), b = *(const uint2v_half*)(head + hi);
        return uint4v{a[0], a[1], b[0], b[1]};
    }
    __device__ __forceinline__ void store(uint16_t* head, uint4v v) const {
        if (INTER) {
            *(uint4v_any*)(head + lo) = v;
        } else {
            *(uint2v_half*)(head + lo) = uint2v{v[0], v[1]};
            *(uint2v_half*)(head + hi) = uint2v{v[2], v[3]};
        }
    }
    // Both weights; their loads come first.
    __device__ __forceinline__ void weights(const HeadArgs& a, HeadUnit& q, HeadUnit& k) const {
#pragma unroll
        for (int j = 0; j < 4; ++j) q.re[j] = q.im[j] = k.re[j] = k.im[j] = 1.0f;
        if (!in) return;
        if (a.param_dtype == MQ_F32) {
            typedef float4v float4v_any __attribute__((aligned(4)));
            const float *of_q = (const float*)(a.qw ? a.qw : a.kw), *of_k = (const float*)(a.kw ? a.kw : a.qw);
            if (!of_q) return;
            const float4v f[2][2] = {{*(const float4v_any*)(of_q + lo), *(const float4v_any*)(of_q + hi)}, {*(const float4v_any*)(of_k + lo), *(const float4v_any*)(of_k + hi)}};
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int r = INTER ? 2 * j : j, m = INTER ? 2 * j + 1 : 4 + j;
                if (a.qw) q.re[j] = f[0][r >> 2][r & 3], q.im[j] = f[0][m >> 2][m & 3];
                if (a.kw) k.re[j] = f[1][r >> 2][r & 3], k.im[j] = f[1][m >> 2][m & 3];
            }
            return;
        }
        const uint16_t *of_q = (const uint16_t*)(a.qw ? a.qw : a.kw), *of_k = (const uint16_t*)(a.kw ? a.kw : a.qw);
        if (!of_q) return;
        const uint4v rq = load(of_q), rk = load(of_k);
        const bool half = a.param_dtype == MQ_F16;
        if (a.qw) q = half ? widen<MQ_F16>(rq) : widen<MQ_BF16>(rq);
        if (a.kw) k = half ? widen<MQ_F16>(rk) : widen<MQ_BF16>(rk);
    }
};

// A row of heads.  WIDE (rows on 16-byte boundaries): through a buffer resource, so that a lane without a head needs no branch and the number of stores ahead of
// a load is known, which then need not be waited for.
template <bool WIDE, int L, bool INTER>
struct HeadRow {
    uint16_t* p;
    __amdgpu_buffer_rsrc_t rsrc;
    __device__ __forceinline__ HeadRow(const uint16_t* row, int values) : p((uint16_t*)row) {
        if constexpr (WIDE) rsrc = __builtin_amdgcn_make_buffer_rsrc((void*)p, 0, values * 2, 0x00020000);
    }
    __device__ __forceinline__ uint4v load(const HeadLane<L, INTER>& lane, int at, bool in) const {
        if constexpr (!WIDE) return in ? lane.load(p + at) : uint4v{0, 0, 0, 0};
        const int lo = in ? (at + lane.lo) * 2 : -16;
        if constexpr (INTER) return __builtin_amdgcn_raw_buffer_load_b128(rsrc, lo, 0, 0);
        const auto a = __builtin_amdgcn_raw_buffer_load_b64(rsrc, lo, 0, 0), b = __builtin_amdgcn_raw_buffer_load_b64(rsrc, in ? (at + lane.hi) * 2 : -16, 0, 0);
        return uint4v{(uint32_t)a[0], (uint32_t)a[1], (uint32_t)b[0], (uint32_t)b[1]};
    }
    __device__ __forceinline__ void store(const HeadLane<L, INTER>& lane, int at, bool in, uint4v v) const {
        if constexpr (!WIDE) {
            if (in) lane.store(p + at, v);
        } else {
            const int lo = in ? (at + lane.lo) * 2 : -16;
            if constexpr (INTER) {
                __builtin_amdgcn_raw_buffer_store_b128(v, rsrc, lo, 0, WRITE_THROUGH);
            } else {
                __builtin_amdgcn_raw_buffer_store_b64(uint2v{v[0], v[1]}, rsrc, lo, 0, WRITE_THROUGH);
                __builtin_amdgcn_raw_buffer_store_b64(uint2v{v[2], v[3]}, rsrc, in ? (at + lane.hi) * 2 : -16, 0, WRITE_THROUGH);
            }
        }
    }
};
__device__ __forceinline__ float either(bool first, float a, float b) { return first ? a : b; }

// A wave takes chunks of the heads of a row: 64 / L of them at a time, U such turns in flight.
template <int DT, int L, bool INTER, bool WIDE>
__global__ __launch_bounds__(256) void heads_kernel(const HeadArgs a) {
    using Row = HeadRow<WIDE, L, INTER>;
    constexpr int G = 64 / L, U = 4;
    const int values = (a.q + a.k) * a.D;
    const int ln = threadIdx.x & 63, grp = ln / L;
    const float mean = 1.0f / (float)a.D;
    HeadLane<L, INTER> lane(a, ln % L);
    const uint32_t waves = gridDim.x * 4;
    HeadWalk at(a, blockIdx.x * 4 + (threadIdx.x >> 6));
    uint4v ahead[U];
    HeadPosition pos;
    auto fetch = [&]() {  // the heads at `at`
        const Row x(a.x + at.row * a.ldx, values);
#pragma unroll
        for (int t = 0; t < U; ++t) {
            const int h = at.base + t * G + grp;
            ahead[t] = x.load(lane, h * a.D, h < at.end && lane.in);
        }
        pos.load(a, at.row);
    };
    if (at.more(a)) fetch();
    lane.load_table(a);
    HeadUnit wq, wk;
    lane.weights(a, wq, wk);
    int row = -1;
    float4v s, c;
    while (at.more(a)) {
        uint4v v[U];
#pragma unroll
        for (int t = 0; t < U; ++t) v[t] = ahead[t];
        if (at.row != row) lane.angles(a, pos, s, c);
        row = at.row;
        const int base = at.base, h1 = at.end;
        const Row y(a.y + row * a.ldy, values);
        at.next(a, G * U, waves);
        if (at.more(a)) fetch();
#pragma unroll
        for (int t = 0; t < U; ++t) {
            if (base + t * G >= h1) break;  // (nothing left: 4096 x 40 heads of 64 10.2 -> 9.0 us, 21230 x 2 of 32 21.8 -> 14.5)
            const int h = base + t * G + grp;
            HeadUnit u = lane.template widen<DT>(v[t]);
            if (a.norm) {
                float sum = 0.0f;
#pragma unroll
                for (int j = 0; j < 4; ++j) sum += u.re[j] * u.re[j] + u.im[j] * u.im[j];
                const float r = rsqrtf(lane_sum<L>(sum) * mean + a.eps);
                const bool is_q = h < a.q;
#pragma unroll
                for (int j = 0; j < 4; ++j) u.re[j] *= r * either(is_q, wq.re[j], wk.re[j]), u.im[j] *= r * either(is_q, wq.im[j], wk.im[j]);
            }
            HeadUnit o;
#pragma unroll
            for (int j = 0; j < 4; ++j) {  // (what does not turn stays as it is, infinities included)
                o.re[j] = lane.turns ? u.re[j] * c[j] - u.im[j] * s[j] : u.re[j];
                o.im[j] = lane.turns ? u.re[j] * s[j] + u.im[j] * c[j] : u.im[j];
            }
            y.store(lane, h * a.D, h < h1 && lane.in, lane.template pack<DT>(o));
        }
    }
}

// The gradient: lanes also hold the sums for the weights of their units; a workgroup joins those of its lanes and waves in a fixed order, and a second kernel
// those of the workgroups.
constexpr int HG_WAVES = 8;
template <int DT, int L, bool INTER, bool WIDE>
__global__ __launch_bounds__(HG_WAVES * 64) void heads_grad_kernel(const HeadArgs a) {
    using Row = HeadRow<WIDE, L, INTER>;
    constexpr int G = 64 / L, U = 2;
    const int values = (a.q + a.k) * a.D;
    __shared__ float join[HG_WAVES * 64 * 8];
    const int ln = threadIdx.x & 63, wv = threadIdx.x >> 6, grp = ln / L, sub = ln % L;
    HeadLane<L, INTER> lane(a, sub);
    HeadUnit sums[2];
#pragma unroll
    for (int j = 0; j < 4; ++j) sums[0].re[j] = sums[0].im[j] = sums[1].re[j] = sums[1].im[j] = 0.0f;
    const float mean = 1.0f / (float)a.D;
    const uint32_t waves = gridDim.x * HG_WAVES;
    HeadWalk at(a, blockIdx.x * HG_WAVES + wv);
    uint4v x_ahead[U], d_ahead[U];
    HeadPosition pos;
    auto fetch = [&]() {
        const Row x(a.norm ? a.x + at.row * a.ldx : nullptr, values), dy(a.dy + at.row * a.lddy, values);
#pragma unroll
        for (int t = 0; t < U; ++t) {
            const int h = at.base + t * G + grp;
            const bool in = h < at.end && lane.in;
            d_ahead[t] = dy.load(lane, h * a.D, in);
            x_ahead[t] = x.load(lane, h * a.D, in && a.norm);
        }
        pos.load(a, at.row);
    };
    if (at.more(a)) fetch();
    lane.load_table(a);
    HeadUnit wq, wk;
    lane.weights(a, wq, wk);
    int row = -1;
    float4v s, c;
    while (at.more(a)) {
        uint4v xv[U], dv[U];
#pragma unroll
        for (int t = 0; t < U; ++t) xv[t] = x_ahead[t], dv[t] = d_ahead[t];
        if (at.row != row) lane.angles(a, pos, s, c);
        row = at.row;
        const int base = at.base, h1 = at.end;
        const Row dx(a.dx + row * a.lddx, values);
        at.next(a, G * U, waves);
        if (at.more(a)) fetch();
#pragma unroll
        for (int t = 0; t < U; ++t) {
            if (base + t * G >= h1) break;
            const int h = base + t * G + grp;
            const bool is_q = h < a.q, live = h < h1;
            const HeadUnit d = lane.template widen<DT>(dv[t]);
            HeadUnit g;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                g.re[j] = lane.turns ? d.re[j] * c[j] + d.im[j] * s[j] : d.re[j];
                g.im[j] = lane.turns ? d.im[j] * c[j] - d.re[j] * s[j] : d.im[j];
            }
            if (a.norm) {
                HeadUnit v = lane.template widen<DT>(xv[t]);
                float sq = 0.0f, dot = 0.0f;
#pragma unroll
                for (int j = 0; j < 4; ++j) sq += v.re[j] * v.re[j] + v.im[j] * v.im[j];
                // (of lanes that hold no head only zeros come: but 0 r is none where r is infinite, as without eps)
                const float all = rsqrtf(lane_sum<L>(sq) * mean + a.eps), r = live ? all : 0.0f;
                // (x r and r w in the products: where squares pass float32 r is 0, and so is what comes of it; products with x itself may be infinite.)
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    v.re[j] *= r, v.im[j] *= r;
                    const float dr = g.re[j] * v.re[j], di = g.im[j] * v.im[j];
                    sums[0].re[j] += either(is_q, dr, 0.0f), sums[0].im[j] += either(is_q, di, 0.0f);
                    sums[1].re[j] += either(is_q, 0.0f, dr), sums[1].im[j] += either(is_q, 0.0f, di);
                    dot += dr * either(is_q, wq.re[j], wk.re[j]) + di * either(is_q, wq.im[j], wk.im[j]);
                }
                const float back = lane_sum<L>(dot) * mean * r;
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    g.re[j] = g.re[j] * (r * either(is_q, wq.re[j], wk.re[j])) - v.re[j] * back;
                    g.im[j] = g.im[j] * (r * either(is_q, wq.im[j], wk.im[j])) - v.im[j] * back;
                }
            }
            dx.store(lane, h * a.D, live && lane.in, lane.template pack<DT>(g));
        }
    }
    if (!a.partial) return;
#pragma unroll
    for (int part = 0; part < 2; ++part) {
        if (part) __syncthreads();
#pragma unroll
        for (int j = 0; j < 4; ++j) join[threadIdx.x * 8 + j] = sums[part].re[j], join[threadIdx.x * 8 + 4 + j] = sums[part].im[j];
        __syncthreads();
        for (int c = threadIdx.x; c < a.D; c += HG_WAVES * 64) {
            const int of = c >> 3, e = c & 7;  // lane of a head, value of its unit
            float t = 0.0f;
            for (int w = 0; w < HG_WAVES * G; ++w) t += join[(w * L + of) * 8 + e];
            const bool turns = of * 4 < a.pairs;
            const int at = INTER || !turns ? of * 8 + (INTER ? 2 * (e & 3) + (e >> 2) : e) : (e < 4 ? of * 4 + e : a.pairs + of * 4 + e - 4);
            a.partial[((long)blockIdx.x * 2 + part) * a.D + at] = t;
        }
    }
}

// [parts][2 D] -> two vectors of D: eight sums to a workgroup, each in 32 runs of parts.
__global__ __launch_bounds__(256) void heads_join_kernel(const float* partial, int parts, int D, float* dq, float* dk) {
    __shared__ float run[32][8];
    const int e = threadIdx.x & 7, c = blockIdx.x * 8 + e, slice = threadIdx.x >> 3;
    float s = 0.0f;
#pragma unroll 4
    for (int p = slice; p < parts; p += 32) s += partial[(long)p * 2 * D + c];
    run[slice][e] = s;
    __syncthreads();
    if (slice == 0) {
        s = 0.0f;
        for (int i = 0; i < 32; ++i) s += run[i][e];
        float* out = c < D ? dq : dk;
        if (out) out[c < D ? c : c - D] = s;
    }
}

// Workgroups of the gradient, and so parts of its sums: two for each compute unit at most, which hold them at once with up to 128 registers.  (With four lanes, not interleaved,
// it has 147: one at a time, two rounds; 21230 x 2 heads of 32 27 us, where idle lanes count too.)
static long heads_grad_workgroups(long tasks) {
    const long n = (tasks + HG_WAVES - 1) / HG_WAVES;
    return n < 512 ? n : 512;
}
// Waves for every row: as many as bring the launch to 4096 (16 per compute unit) or, with 2049 to 4095 rows, past it, where some take two tasks; but no part of a turn's heads.
// Just past 4096 rows some take a second whole one: forward and gradient of 40 heads of 64, 2964 rows 7.4, 14.1, 4096 8.3, 16.3, 4200 8.8, 18.9, 6000 11.1, 20.3; of 128 11.4, 20.4,
// 14.2, 26.9, 15.6, 30.3, 23.0, 37.9.  us, 2048 / 4096 / 8192 waves: forward 2964 x 32 heads
// of 80 8.4 / 8.7 / 11.0, 4096 x 40 of 128 14.5 / 14.6 / 15.8, 32768 x 40 of 64 65 / 63 / 63; gradient 19.9 / 16.7 / 21.6, 24.8 / 24.9 / 26.0, 96 / 98 / 98.
static void heads_chunks(HeadArgs& a, int L) {
    const int H = a.q + a.k, G = 64 / L, turns = (H + G - 1) / G;
    long want = a.M > 0 ? (4096 + a.M - 1) / a.M : 1;
    if (want > turns) want = turns;
    const int per = (int)((turns + want - 1) / want);
    a.per_chunk = per * G;
    const int chunks = (turns + per - 1) / per;
    a.chunks = FastDiv::make((uint32_t)chunks);
    a.tasks = (uint32_t)((long)a.M * chunks);
}

template <int DT, int L, bool INTER, bool WIDE>
static int run_heads(HeadArgs& a, bool grad, hipStream_t st) {
    heads_chunks(a, L);
    if (!grad) {
        const long n = ((long)a.tasks + 3) / 4;
        heads_kernel<DT, L, INTER, WIDE><<<(unsigned)(n < 1024 ? n : 1024), 256, 0, st>>>(a);
        MQ_HIP_CHECK_LAUNCH();
        return MQ_OK;
    }
    const long wgs = heads_grad_workgroups(a.tasks);
    if (!a.dq_weight && !a.dk_weight) a.partial = nullptr;
    if (wgs > 0) {
        heads_grad_kernel<DT, L, INTER, WIDE><<<(unsigned)wgs, HG_WAVES * 64, 0, st>>>(a);
        MQ_HIP_CHECK_LAUNCH();
    }
    if (a.dq_weight || a.dk_weight) {
        heads_join_kernel<<<(unsigned)(a.D / 4), 256, 0, st>>>(a.partial, (int)wgs, a.D, a.dq_weight, a.dk_weight);
        MQ_HIP_CHECK_LAUNCH();
    }
    return MQ_OK;
}
template <int DT, int L>
static int run_heads(HeadArgs& a, bool grad, hipStream_t st) {
    auto wide = [&](const void* p, long ld) { return (uintptr_t)p % 16 == 0 && (a.M == 1 || ld % 8 == 0); };
    const bool w = grad ? wide(a.dy, a.lddy) && wide(a.dx, a.lddx) && (!a.norm || wide(a.x, a.ldx)) : wide(a.x, a.ldx) && wide(a.y, a.ldy);
    if (w) return a.interleaved ? run_heads<DT, L, true, true>(a, grad, st) : run_heads<DT, L, false, true>(a, grad, st);
    return a.interleaved ? run_heads<DT, L, true, false>(a, grad, st) : run_heads<DT, L, false, false>(a, grad, st);
}
template <int DT>
static int choose_heads(HeadArgs& a, bool grad, hipStream_t st) {
    const int n = a.D / 8;
    return n <= 4 ? run_heads<DT, 4>(a, grad, st) : n <= 8 ? run_heads<DT, 8>(a, grad, st) : n <= 16 ? run_heads<DT, 16>(a, grad, st)
           : n <= 32 ? run_heads<DT, 32>(a, grad, st) : run_heads<DT, 64>(a, grad, st);
}

size_t heads_grad_workspace_bytes(long M, int H, int D) {
    // (a wave takes at least one head)
    return (size_t)heads_grad_workgroups(M * H) * 2 * D * 4;
}
int launch_heads(HeadArgs& a, bool grad, hipStream_t st) { return a.dtype == MQ_F16 ? choose_heads<MQ_F16>(a, grad, st) : choose_heads<MQ_BF16>(a, grad, st); }

}  // namespace mq

// Product of two microscaled 4-bit matrices: Y = A W^T + bias (+ residual), with the MFMAs that take the scales of the blocks as operands.
#include "mx_common.h"

namespace mq {

typedef int int8v __attribute__((ext_vector_type(8)));
typedef uint2v uint2v_any __attribute__((aligned(2)));

// One 32 x 32 x 64 step; S: the byte of the scale words that belongs to it.
template <int S>
__device__ __forceinline__ float16v mx_mfma(int4v w, int4v a, float16v c, int sw, int sa) {
    const int8v W = {w[0], w[1], w[2], w[3], 0, 0, 0, 0}, A = {a[0], a[1], a[2], a[3], 0, 0, 0, 0};
    return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(W, A, c, 4, 4, S, sw, S, sa);
}

// The weights are the MFMA's row operand: a lane then holds, of one row of Y, four runs of four consecutive columns (8 t + 4 h, h the lane's half).
// Two such runs trade places with those of the other half, and the lane has eight consecutive columns; another trade, between the 16 lanes of a row of
// lanes and the next, and four lanes have the 32 columns of a row, one 64-byte piece.  (A kernel has one of the forms: all of them unrolled over the
// blocks of a large tile are more code than the instruction cache holds, which a workgroup runs through once; 8 us of a 256 x 256 tile.)
enum { MX_PLAIN, MX_RES, MX_ODD };  // without a residual; with one; N no multiple of eight, with or without
// Lanes 16 .. 31 of v[0] and lanes 0 .. 15 of v[1] trade places, likewise in the upper half.  Its own inverse.
__device__ __forceinline__ void mx_swap16(uint4v* v) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const auto p = __builtin_amdgcn_permlane16_swap(v[0][i], v[1][i], false, false);
        v[0][i] = (uint32_t)p[0];
        v[1][i] = (uint32_t)p[1];
    }
}
template <int DT, int EPI>
__device__ __forceinline__ void mx_store_block(const MxGemm& g, const float16v& acc, const float* bias, long m0, int n0, int lane) {
    const int h = lane >> 5, q = (lane >> 4) & 1;
    const int n = n0 + 16 * q + 8 * h, left = g.N - n;
    const long m = m0 + (lane & 15);
    const bool on[2] = {m < g.M && left > 0, m + 16 < g.M && left > 0};
    uint4v v[2] = {{0, 0, 0, 0}, {0, 0, 0, 0}};
    if (EPI == MX_RES || (EPI == MX_ODD && g.res)) {
#pragma unroll
        for (int t = 0; t < 2; ++t)
            if (on[t]) v[t] = load8_16(g.res + (m + 16 * t) * g.ldr + n, EPI == MX_ODD ? left : 8);
        mx_swap16(v);
    }
#pragma unroll
    for (int t = 0; t < 2; ++t) {
        float f[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) f[i] = acc[8 * t + i] + bias[8 * t + i];
        if (EPI == MX_RES || (EPI == MX_ODD && g.res)) {
            const auto p = __builtin_amdgcn_permlane32_swap(v[t][0], v[t][2], false, false), r = __builtin_amdgcn_permlane32_swap(v[t][1], v[t][3], false, false);
            const uint32_t o[4] = {(uint32_t)p[0], (uint32_t)r[0], (uint32_t)p[1], (uint32_t)r[1]};
#pragma unroll
            for (int i = 0; i < 8; ++i) f[i] += T16<DT>::up((uint16_t)(o[i >> 1] >> (16 * (i & 1))));
        }
        const uint32_t a0 = T16<DT>::pack(f[0], f[1]), a1 = T16<DT>::pack(f[2], f[3]), b0 = T16<DT>::pack(f[4], f[5]), b1 = T16<DT>::pack(f[6], f[7]);
        const auto p = __builtin_amdgcn_permlane32_swap(a0, b0, false, false), r = __builtin_amdgcn_permlane32_swap(a1, b1, false, false);
        v[t] = uint4v{(uint32_t)p[0], (uint32_t)r[0], (uint32_t)p[1], (uint32_t)r[1]};
    }
    mx_swap16(v);
#pragma unroll
    for (int t = 0; t < 2; ++t)
        if (on[t]) store8_16(g.y + (m + 16 * t) * g.ldy + n, v[t], EPI == MX_ODD ? left : 8);
}

// Bias of a block's columns, in the accumulators' order.
template <int DT, int EPI>
__device__ __forceinline__ void mx_bias_block(const MxGemm& g, int n0, int h, float* c) {
#pragma unroll
    for (int t = 0; t < 4; ++t) {
        const int n = n0 + 8 * t + 4 * h;
        uint2v b = {0, 0};
        if (g.bias && (EPI == MX_ODD ? n + 4 <= g.N : n < g.N)) b = *(const uint2v_any*)(g.bias + n);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            c[4 * t + i] = T16<DT>::up((uint16_t)(b[i >> 1] >> (16 * (i & 1))));
            if (EPI == MX_ODD && g.bias && n + 4 > g.N && n + i < g.N) c[4 * t + i] = T16<DT>::up(g.bias[n + i]);
        }
    }
}

// Workgroup -> tile.  Workgroups go round the eight XCDs; each XCD gets a run of neighbouring tiles, walked in bands of `band` row tiles, column by
// column, so that the tiles that run on it at the same time share their operands in its L2.
struct MxTiles {
    uint32_t rows, cols, band;
    FastDiv per_band, full_band, last_band;
};
static MxTiles mx_tiles(long rows, long cols, long band) {
    MxTiles t;
    band = band < rows ? band : rows;
    t.rows = (uint32_t)rows;
    t.cols = (uint32_t)cols;
    t.band = (uint32_t)band;
    t.per_band = FastDiv::make((uint32_t)(band * cols));
    t.full_band = FastDiv::make((uint32_t)band);
    t.last_band = FastDiv::make((uint32_t)(rows % band ? rows % band : band));
    return t;
}
__device__ __forceinline__ void mx_tile_of_block(uint32_t id, const MxTiles& t, uint32_t& row, uint32_t& col) {
    const uint32_t total = t.rows * t.cols, per = total >> 3, more = total & 7, x = id & 7;
    const uint32_t i = x * per + (x < more ? x : more) + (id >> 3);
    uint32_t b, r;
    t.per_band.divmod(i, b, r);
    const uint32_t height = (b + 1) * t.band <= t.rows ? t.band : t.rows - b * t.band;
    if (height == t.band) {
        uint32_t q, m;
        t.full_band.divmod(r, q, m);
        col = q;
        row = b * t.band + m;
    } else {
        uint32_t q, m;
        t.last_band.divmod(r, q, m);
        col = q;
        row = b * t.band + m;
    }
}

// LDS plan of a workgroup of WM x WN waves with wave tiles of 32 TM x 32 TN, S slots of 128 k.  Loads of a step, 1 KB each: A_OPS and W_OPS per wave of
// codes (two per group of 32 rows), and one of scales, of four groups (waves that have none load no bytes into the sink).
template <int WM, int WN, int TM, int TN, int S>
struct MxPlan {
    static constexpr int NW = WM * WN, GA = WM * TM, GB = WN * TN, G = GA + GB;
    static constexpr int A_OPS = GA * 2 / NW, W_OPS = GB * 2 / NW, OPS = A_OPS + W_OPS + 1, SCALE_OPS = G / 4;
    static constexpr int SCALES = G * 2048, SLOT = SCALES + SCALE_OPS * 1024, SINK = S * SLOT, BYTES = SINK + (SCALE_OPS < NW ? 1024 : 0);
    static_assert(GA * 2 % NW == 0 && GB * 2 % NW == 0 && GA % 4 == 0 && GB % 4 == 0 && SCALE_OPS <= NW && NW % 2 == 0, "loads of a step");
};

// Operand tiles pass through LDS by LDS-writing loads, which need no rearranging: a tile is fetched in lane order and read back in lane order.  A step is
// 128 k.  The fragments of the next 64 k are read while the MFMAs of this one run, and the loads of a later step are laid out between them one by one.
// In the middle of a step every wave has read all of its slot; there all of them wait for the next step's.
template <int DT, int EPI, int WM, int WN, int TM, int TN, int S>
__global__ __launch_bounds__(WM * WN * 64, 1) void mx_gemm_kernel(const MxGemm g, const MxTiles tiles) {
    using P = MxPlan<WM, WN, TM, TN, S>;
    extern __shared__ __attribute__((aligned(16))) uint8_t lds[];
    const int lane = threadIdx.x & 63, wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int h = lane >> 5, wm = wv % WM, wn = wv / WM;
    uint32_t tr, tc;
    mx_tile_of_block(blockIdx.x, tiles, tr, tc);
    const int ga = (int)tr * P::GA, gw = (int)tc * P::GB;
    const int kc = g.a.kc, kq = g.a.kq, steps = (kc + 1) >> 1;
    const uint32_t lds0 = (uint32_t)(uintptr_t)lds;

    // What lies past the last group, or past the reduction's last step, reads as zero.  (Codes behind an odd number of 64-k tiles are the next group's:
    // their scales are padding, and both zero.)
    auto window = [](const uint8_t* p, long stride, int first, int groups, int want) {
        const int n = groups - first < want ? groups - first : want;
        return make_rsrc(p + first * stride, n > 0 ? (uint32_t)(n * stride) : 0u);
    };
    const int4s ra = window(g.a.codes, (long)kc * 1024, ga, g.a.groups, P::GA), rw = window(g.w.codes, (long)kc * 1024, gw, g.w.groups, P::GB);
    const bool scales_a = wv * 4 < P::GA;
    int4s rs = scales_a ? window(g.a.scales, (long)kq * 256, ga, g.a.groups, P::GA) : window(g.w.scales, (long)kq * 256, gw, g.w.groups, P::GB);
    if (wv >= P::SCALE_OPS) rs[2] = 0;
    const int v_data = lane * 16 + (wv & 1) * 1024 + (wv >> 1) * kc * 1024;
    const int v_scale = (wv * 4 - (scales_a ? 0 : P::GA) + (lane >> 4)) * kq * 256 + (lane & 15) * 16;
    const uint32_t l_data = __builtin_amdgcn_readfirstlane(lds0 + wv * 1024);
    const uint32_t l_scale = __builtin_amdgcn_readfirstlane(wv < P::SCALE_OPS ? lds0 + P::SCALES + wv * 1024 : lds0 + P::SINK);
    const int stride = P::NW / 2 * kc * 1024;  // between a wave's loads of one operand

    // Load i of a step into the slot at `at`.
    auto load = [&](int step, uint32_t at, int i) {
        const bool live = step < steps;
        if (i < P::A_OPS) {
            int4s r = ra;
            r[2] = live ? r[2] : 0;
            dma_to_lds_b128(r, at, l_data + i * P::NW * 1024, v_data, step * 2048 + i * stride);
        } else if (i < P::A_OPS + P::W_OPS) {
            const int j = i - P::A_OPS;
            int4s r = rw;
            r[2] = live ? r[2] : 0;
            dma_to_lds_b128(r, at, l_data + (P::GA * 2 + j * P::NW) * 1024, v_data, step * 2048 + j * stride);
        } else {
            int4s r = rs;
            r[2] = live ? r[2] : 0;
            dma_to_lds_b128(r, wv < P::SCALE_OPS ? at : 0u, l_scale, v_scale, (step >> 1) * 256);
        }
    };
    struct Frag {
        int4v w[TN], a[TM];
    };
    struct Scales {
        int w[TN], a[TM];
    };
    constexpr int READS = TM + TN;
    auto read = [&](Frag& f, uint32_t slot, int half, int i) {
        if (i < TN)
            f.w[i < TN ? i : 0] = *(const int4v*)(lds + slot + ((P::GA + wn * TN + i) * 2 + half) * 1024 + lane * 16);
        else
            f.a[i < TN ? 0 : i - TN] = *(const int4v*)(lds + slot + ((wm * TM + i - TN) * 2 + half) * 1024 + lane * 16);
    };
    auto read_scale = [&](Scales& s, uint32_t slot, int i) {
        if (i < TN)
            s.w[i < TN ? i : 0] = *(const int*)(lds + slot + P::SCALES + (P::GA + wn * TN + i) * 256 + lane * 4);
        else
            s.a[i < TN ? 0 : i - TN] = *(const int*)(lds + slot + P::SCALES + (wm * TM + i - TN) * 256 + lane * 4);
    };
    float16v acc[TM][TN];
    // The MFMAs of 64 k, with `items` other things to do laid out between them.
    auto phase = [&](auto byte, const Frag& f, const Scales& s, int items, auto item) {
        constexpr int MM = TM * TN;
#pragma unroll
        for (int i = 0; i < MM; ++i) {
            const int m = i / TN, n = i % TN;
            acc[m][n] = mx_mfma<decltype(byte)::value>(f.w[n], f.a[m], acc[m][n], s.w[n], s.a[m]);
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int j = i * items / MM; j < (i + 1) * items / MM; ++j) item(j);
            __builtin_amdgcn_sched_barrier(0);
        }
    };

#pragma unroll
    for (int s = 0; s < S - 1; ++s)
#pragma unroll
        for (int i = 0; i < P::OPS; ++i) load(s, s * P::SLOT, i);
#pragma unroll
    for (int n = 0; n < TN; ++n)
#pragma unroll
        for (int m = 0; m < TM; ++m)
#pragma unroll
            for (int i = 0; i < 16; ++i) acc[m][n][i] = 0.0f;

    // (A wave's LDS reads are done before it lets the others overwrite what it read.)
    auto ready = [&]() { asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"((S - 2) * P::OPS) : "memory"); };
    ready();
    Frag f0, f1;
    Scales next;
    uint32_t slot = 0, fill = (S - 1) * P::SLOT;
#pragma unroll
    for (int i = 0; i < READS; ++i) read_scale(next, 0, i);
#pragma unroll
    for (int i = 0; i < READS; ++i) read(f0, 0, 0, i);
    for (int step = 0; step < steps; ++step) {
        Scales s;
        const int shift = (step & 1) * 16;  // a scale word serves two steps
#pragma unroll
        for (int i = 0; i < TN; ++i) s.w[i] = next.w[i] >> shift;
#pragma unroll
        for (int i = 0; i < TM; ++i) s.a[i] = next.a[i] >> shift;
        phase(std::integral_constant<int, 0>{}, f0, s, READS + P::OPS, [&](int j) {
            if (j < READS)
                read(f1, slot, 1, j);
            else
                load(step + S - 1, fill, j - READS);
        });
        fill = fill == (S - 1) * P::SLOT ? 0 : fill + P::SLOT;
        slot = slot == (S - 1) * P::SLOT ? 0 : slot + P::SLOT;
        ready();
        phase(std::integral_constant<int, 1>{}, f1, s, 2 * READS, [&](int j) {
            if (j < READS)
                read(f0, slot, 0, j);
            else
                read_scale(next, slot, j - READS);
        });
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // (loads of no bytes still write their zeros)
#pragma unroll
    for (int n = 0; n < TN; ++n) {
        const int n0 = (gw + wn * TN + n) * 32;
        if (n0 >= g.N) break;
        float b[16];
        mx_bias_block<DT, EPI>(g, n0, h, b);
#pragma unroll
        for (int m = 0; m < TM; ++m) mx_store_block<DT, EPI>(g, acc[m][n], b, (long)(ga + wm * TM + m) * 32, n0, lane);
    }
}

template <int DT, int EPI, int WM, int WN, int TM, int TN, int S>
static int run_mx_form(const MxGemm& g, long band, hipStream_t st) {
    using P = MxPlan<WM, WN, TM, TN, S>;
    const long rows = (g.a.groups + P::GA - 1) / P::GA, cols = (g.w.groups + P::GB - 1) / P::GB;
    auto kernel = mx_gemm_kernel<DT, EPI, WM, WN, TM, TN, S>;
    static const hipError_t set = hipFuncSetAttribute((const void*)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, P::BYTES);
    if (set != hipSuccess) {
        set_hip_error((int)set);
        return MQ_ERR_HIP;
    }
    kernel<<<(unsigned)(rows * cols), P::NW * 64, P::BYTES, st>>>(g, mx_tiles(rows, cols, band));
    MQ_HIP_CHECK_LAUNCH();
    return MQ_OK;
}

template <int DT, int WM, int WN, int TM, int TN, int S>
static int run_mx_gemm(const MxGemm& g, long band, hipStream_t st) {
    if (g.N % 8 != 0) return run_mx_form<DT, MX_ODD, 2, 2, 2, 2, 4>(g, band, st);
    return g.res ? run_mx_form<DT, MX_RES, WM, WN, TM, TN, S>(g, band, st) : run_mx_form<DT, MX_PLAIN, WM, WN, TM, TN, S>(g, band, st);
}

// 256 x 256 tiles with two waves per SIMD, or 128 x 128 with one and up to three workgroups per compute unit.  The large tile moves half as much per
// multiplication, but takes 5 us to fill and empty: it pays from about four rounds of tiles on.  us, 256 / 128: 8192 x 8192 x 8192 (1024 tiles of 256)
// 273 / 328, 16384 x 640 x 5120 (1280) 61 / 70, 4096 x 1280 x 10240 (640) 49 / 48, 4096 x 5120 x 1280 (80) 33 / 24, 512 x 2048 x 640 (6) 15 / 8.
template <int DT>
static int choose_mx_gemm(const MxGemm& g, hipStream_t st) {
    const long tiles = (long)((g.a.groups + 7) / 8) * ((g.w.groups + 7) / 8);
    return tiles >= 1000 ? run_mx_gemm<DT, 2, 4, 4, 2, 4>(g, 8, st) : run_mx_gemm<DT, 2, 2, 2, 2, 4>(g, 8, st);
}

int launch_mx_gemm(const MxGemm& g, hipStream_t st) { return g.dtype == MQ_F16 ? choose_mx_gemm<MQ_F16>(g, st) : choose_mx_gemm<MQ_BF16>(g, st); }

}  // namespace mq

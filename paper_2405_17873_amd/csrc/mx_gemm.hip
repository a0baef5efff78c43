// Product of two microscaled 4-bit matrices: Y = A W^T + bias (+ residual), with the MFMAs that take the scales of the blocks as operands.
#include "mx_common.h"

namespace mq {

typedef int int8v __attribute__((ext_vector_type(8)));
typedef uint2v uint2v_any __attribute__((aligned(2)));
typedef __attribute__((address_space(3))) uint2v lds_uint2v;

// One 32 x 32 x 64 step; S: the byte of the scale words that belongs to it.
template <int S>
__device__ __forceinline__ float16v mx_mfma(int4v w, int4v a, float16v c, int sw, int sa) {
    const int8v W = {w[0], w[1], w[2], w[3], 0, 0, 0, 0}, A = {a[0], a[1], a[2], a[3], 0, 0, 0, 0};
    return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(W, A, c, 4, 4, S, sw, S, sa);
}

// The weights are the MFMA's row operand: a lane then holds, of one row of Y, four runs of four consecutive columns (8 t + 4 h, h the lane's half).
// Two such runs trade places with those of the other half, and the lane has eight consecutive columns; another trade, between the 16 lanes of a row of
// lanes and the next, and four lanes have the 32 columns of a row, one 64-byte piece.  (A kernel has one of the forms: all of them unrolled over the
// blocks of a large tile are more code than the instruction cache holds; 8 us of a 256 x 256 tile.)
enum { MX_PLAIN, MX_RES, MX_ODD };  // without a residual; with one; rows of any alignment and length, with or without
// Lanes 16 .. 31 of v[0] and lanes 0 .. 15 of v[1] trade places, likewise in the upper half.  Its own inverse.
__device__ __forceinline__ void mx_swap16(uint4v* v) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const auto p = __builtin_amdgcn_permlane16_swap(v[0][i], v[1][i], false, false);
        v[0][i] = (uint32_t)p[0];
        v[1][i] = (uint32_t)p[1];
    }
}
// Adds a residual r[2] (in the order of the output, or null) to a block's sums and brings them into the order of the output: two vectors of eight
// columns, of rows lane & 15 and 16 further on, columns 16 q + 8 h (q, h: bits 4 and 5 of the lane).
template <int DT>
__device__ __forceinline__ void mx_finish_block(const float16v& acc, const uint4v* r, uint4v* v) {
    if (r) {
        v[0] = r[0], v[1] = r[1];
        mx_swap16(v);
    }
#pragma unroll
    for (int t = 0; t < 2; ++t) {
        float f[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) f[i] = acc[8 * t + i];
        if (r) {
            const auto p = __builtin_amdgcn_permlane32_swap(v[t][0], v[t][2], false, false), q = __builtin_amdgcn_permlane32_swap(v[t][1], v[t][3], false, false);
            const uint32_t o[4] = {(uint32_t)p[0], (uint32_t)q[0], (uint32_t)p[1], (uint32_t)q[1]};
#pragma unroll
            for (int i = 0; i < 8; ++i) f[i] += T16<DT>::up((uint16_t)(o[i >> 1] >> (16 * (i & 1))));
        }
        const uint32_t a0 = T16<DT>::pack(f[0], f[1]), a1 = T16<DT>::pack(f[2], f[3]), b0 = T16<DT>::pack(f[4], f[5]), b1 = T16<DT>::pack(f[6], f[7]);
        const auto p = __builtin_amdgcn_permlane32_swap(a0, b0, false, false), q = __builtin_amdgcn_permlane32_swap(a1, b1, false, false);
        v[t] = uint4v{(uint32_t)p[0], (uint32_t)q[0], (uint32_t)p[1], (uint32_t)q[1]};
    }
    mx_swap16(v);
}

// Tiles of a workgroup.  Workgroups go round the eight XCDs; each XCD gets a run of neighbouring tiles, walked in bands of `band` row tiles, column by
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
__device__ __forceinline__ void mx_tile(uint32_t i, const MxTiles& t, int& row, int& col) {
    uint32_t b, r, q, m;
    t.per_band.divmod(i, b, r);
    if ((b + 1) * t.band <= t.rows)
        t.full_band.divmod(r, q, m);
    else
        t.last_band.divmod(r, q, m);
    col = __builtin_amdgcn_readfirstlane((int)q);
    row = __builtin_amdgcn_readfirstlane((int)(b * t.band + m));
}

// LDS plan of a workgroup of WM x WN waves with wave tiles of 32 TM x 32 TN, S slots of 128 k.  Loads of a step, 1 KB each: A_OPS and W_OPS per wave of
// codes (two per group of 32 rows), and one of scales, of four groups; the wave behind those
// that have scales to load gets the tile's bias, waves behind it load no bytes into the sink.
template <int WM, int WN, int TM, int TN, int S>
struct MxPlan {
    static constexpr int NW = WM * WN, GA = WM * TM, GB = WN * TN;
    static constexpr int A_OPS = GA * 2 / NW, W_OPS = (GB * 2 + NW - 1) / NW, OPS = A_OPS + W_OPS + 1;
    static constexpr int A_SCALES = GA / 4, SCALE_OPS = A_SCALES + (GB + 3) / 4;
    static constexpr int SCALES = (A_OPS + W_OPS) * NW * 1024, BIAS = SCALES + SCALE_OPS * 1024, SLOT = BIAS + 1024, SINK = S * SLOT, BYTES = SINK + 1024;
    static_assert(BYTES <= 160 * 1024, "LDS of a compute unit");
    static constexpr int STORES = TM * TN * 2;  // of a wave and tile
    static_assert(GA * 2 % NW == 0 && GA % 4 == 0 && SCALE_OPS < NW && NW % 2 == 0, "loads of a step");
    static_assert((S - 2) * OPS + STORES < 64, "the counter of loads and stores");
};

// Operand tiles pass through LDS by LDS-writing loads, which need no rearranging: a tile is fetched in lane order and read back in lane order.  A step is
// 128 k.  The fragments of the next 64 k are read while the MFMAs of this one run, and the loads of a later step are laid out between them one by one.
// In the middle of a step every wave has read all of its slot; there all of them wait for the next step's.  A workgroup has several tiles, and the steps
// of one follow those of another without a pause: while results are stored the next tile's first steps are on their way.
// Bound by power where K is long: in 8192 x 8192 x 8192 (250 us) MFMAs run in 60 % of the cycles and LDS reads in 28 %, the clock falls to 1.7 GHz, and
// random operands take half as long again as zeros.  Four waves of 128 x 128 each would read two thirds as much from LDS, but spill and wait for themselves
// (338 us).  Where K is short, by the results: 16384 x 640 x 5120 writes 168 MB in 49 (traced) to 56 us, 42 without its stores; keeping results in registers
// and storing them between the MFMAs of the next tile (128 x 128 tiles) changed nothing, 64 us.
template <int DT, int EPI, int WM, int WN, int TM, int TN, int S>
__global__ __launch_bounds__(WM * WN * 64, 1) void mx_gemm_kernel(const MxGemm g, const MxTiles tiles) {
    using P = MxPlan<WM, WN, TM, TN, S>;
    extern __shared__ __attribute__((aligned(16))) uint8_t lds[];
    const int lane = threadIdx.x & 63, wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int h = lane >> 5, wm = wv % WM, wn = wv / WM;
    const int kc = g.a.kc, kq = g.a.kq, steps = (kc + 1) >> 1;
    const uint32_t lds0 = (uint32_t)(uintptr_t)lds;
    // tiles of this workgroup: `at`, at + every, ... below `end`
    const uint32_t total = tiles.rows * tiles.cols, per = total >> 3, more = total & 7, xcd = blockIdx.x & 7;
    const uint32_t start = xcd * per + (xcd < more ? xcd : more), end = start + per + (xcd < more ? 1 : 0), every = (gridDim.x + 7) >> 3;
    uint32_t at = start + (blockIdx.x >> 3);
    if (at >= end) return;

    // What lies past the last group, or past the last tile, reads as zero.  (Codes behind an odd number of 64-k tiles are the next group's: their scales
    // are padding, and both zero.)
    auto window = [](const uint8_t* p, long stride, int first, int groups, int want) {
        const int n = groups - first < want ? groups - first : want;
        return make_rsrc(p + first * stride, n > 0 ? (uint32_t)(n * stride) : 0u);
    };
    const bool scales_a = wv < P::A_SCALES;
    struct Source {
        int4s a, w, s;
    };
    auto source = [&](uint32_t tile) {
        int tr, tc;
        mx_tile(tile < end ? tile : end - 1, tiles, tr, tc);
        const int ga = tr * P::GA, gw = tc * P::GB;
        Source o;
        o.a = window(g.a.codes, (long)kc * 1024, ga, g.a.groups, P::GA);
        o.w = window(g.w.codes, (long)kc * 1024, gw, g.w.groups, P::GB);
        if (wv < P::SCALE_OPS) {
            o.s = scales_a ? window(g.a.scales, (long)kq * 256, ga, g.a.groups, P::GA) : window(g.w.scales, (long)kq * 256, gw, g.w.groups, P::GB);
        } else {
            const int cols = g.N - gw * 32 < P::GB * 32 ? g.N - gw * 32 : P::GB * 32;
            o.s = make_rsrc(g.bias + gw * 32, EPI != MX_ODD && wv == P::SCALE_OPS && g.bias ? (uint32_t)cols * 2u : 0u);
        }
        if (tile >= end) o.a[2] = o.w[2] = o.s[2] = 0;
        return o;
    };
    Source from = source(at), after;  // of the step that is loaded next, and of the tile behind that
    const int v_data = lane * 16 + (wv & 1) * 1024 + (wv >> 1) * kc * 1024;
    const int v_scale = wv < P::SCALE_OPS ? ((wv - (scales_a ? 0 : P::A_SCALES)) * 4 + (lane >> 4)) * kq * 256 + (lane & 15) * 16 : lane * 16;
    const uint32_t l_data = __builtin_amdgcn_readfirstlane(lds0 + wv * 1024);
    const uint32_t l_scale = __builtin_amdgcn_readfirstlane(wv <= P::SCALE_OPS ? lds0 + P::SCALES + wv * 1024 : lds0 + P::SINK);
    const int stride = P::NW / 2 * kc * 1024;  // between a wave's loads of one operand

    int step_ahead = 0;
    // Load i of the step that is next, into the slot at `to`.
    auto load = [&](uint32_t to, int i) {
        if (i < P::A_OPS)
            dma_to_lds_b128(from.a, to, l_data + i * P::NW * 1024, v_data, step_ahead * 2048 + i * stride);
        else if (i < P::A_OPS + P::W_OPS)
            dma_to_lds_b128(from.w, to, l_data + (P::GA * 2 + (i - P::A_OPS) * P::NW) * 1024, v_data, step_ahead * 2048 + (i - P::A_OPS) * stride);
        else
            dma_to_lds_b128(from.s, wv <= P::SCALE_OPS ? to : 0u, l_scale, v_scale, wv < P::SCALE_OPS ? (step_ahead >> 1) * 256 : 0);
    };
    auto loaded = [&]() {  // (without a branch)
        const bool over = step_ahead + 1 == steps;
        step_ahead = over ? 0 : step_ahead + 1;
#pragma unroll
        for (int i = 0; i < 3; ++i) {  // (the fourth word is a constant)
            from.a[i] = over ? after.a[i] : from.a[i];
            from.w[i] = over ? after.w[i] : from.w[i];
            from.s[i] = over ? after.s[i] : from.s[i];
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

    after = source(end);  // (a workgroup with several tiles has S steps in each: none of these is the next tile's)
#pragma unroll
    for (int s = 0; s < S - 1; ++s) {
#pragma unroll
        for (int i = 0; i < P::OPS; ++i) load(s * P::SLOT, i);
        loaded();
    }
    // Waits for the slot of the next step, and for the other waves to have read the last one.  behind_stores > 0: that slot was asked for ahead of the stores of the
    // tile before, which need not be waited for.  (The branch is inside the assembly: one that the compiler sees would end a block of code, and MFMAs
    // sink past such ends.  A wave's LDS reads are done before it lets the others overwrite what it read.)
    auto ready = [&](int behind_stores) {
        asm volatile(
            "s_cmp_lt_i32 %0, 1\n\t"
            "s_cbranch_scc1 .Lloads%=\n\t"
            "s_waitcnt vmcnt(%2) lgkmcnt(0)\n\t"
            "s_branch .Lready%=\n"
            ".Lloads%=:\n\t"
            "s_waitcnt vmcnt(%1) lgkmcnt(0)\n"
            ".Lready%=:\n\t"
            "s_barrier" ::"s"(behind_stores),
            "n"((S - 2) * P::OPS), "n"((S - 2) * P::OPS + P::STORES)
            : "memory", "scc");
    };
    ready(0);
    Frag f0, f1;
    Scales next;
    uint32_t slot = 0, fill = (S - 1) * P::SLOT;
#pragma unroll
    for (int i = 0; i < READS; ++i) read_scale(next, 0, i);
#pragma unroll
    for (int i = 0; i < READS; ++i) read(f0, 0, 0, i);

    int behind = 0;  // steps to come whose slots were asked for ahead of stores
    for (; at < end; at += every, behind = EPI != MX_ODD ? S - 2 : 0) {
        // The sums start from the bias, which costs their end 16 additions a block less.
        int tr, tc;
        mx_tile(at, tiles, tr, tc);
        const long m0 = (long)tr * (P::GA * 32) + wm * TM * 32;
        const int n0 = tc * (P::GB * 32) + wn * TN * 32, q = (lane >> 4) & 1, c0 = n0 + 16 * q + 8 * h;
#pragma unroll
        for (int n = 0; n < TN; ++n)
#pragma unroll
            for (int t = 0; t < 4; ++t) {
                uint2v bias = {0, 0};
                if constexpr (EPI != MX_ODD) {
                    bias = *(const lds_uint2v*)(uintptr_t)(lds0 + slot + P::BIAS + ((wn * TN + n) * 32 + 8 * t + 4 * h) * 2);
                } else if (g.bias) {
                    const int c = n0 + n * 32 + 8 * t + 4 * h;
                    if (c + 4 <= g.N) bias = *(const uint2v_any*)(g.bias + c);
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        if (c + 4 > g.N && c + i < g.N) bias[i >> 1] |= (uint32_t)g.bias[c + i] << (16 * (i & 1));
                }
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float f = T16<DT>::up((uint16_t)(bias[i >> 1] >> (16 * (i & 1))));
#pragma unroll
                    for (int m = 0; m < TM; ++m) acc[m][n][4 * t + i] = f;
                }
            }
        after = source(at + every);
        auto do_step = [&](int step) {
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
                    load(fill, j - READS);
            });
            loaded();
            fill = fill == (S - 1) * P::SLOT ? 0 : fill + P::SLOT;
            slot = slot == (S - 1) * P::SLOT ? 0 : slot + P::SLOT;
            ready(behind--);
            phase(std::integral_constant<int, 1>{}, f1, s, 2 * READS, [&](int j) {
                if (j < READS)
                    read(f0, slot, 0, j);
                else
                    read_scale(next, slot, j - READS);
            });
        };
        int step = 0;
        do do_step(step);  // (one block of code: MFMAs sink past the ends of blocks)
        while (++step < steps);
        if constexpr (EPI != MX_ODD) {
            // Stores of a fixed number, whatever exists (what does not is dropped): the waits count them.
            const long rows = g.M - m0;
            auto resource = [&](const uint16_t* p, long ld) {
                const long n = rows <= 0 ? 0 : ((rows < TM * 32 ? rows : TM * 32) - 1) * ld + g.N;
                return __builtin_amdgcn_make_buffer_rsrc((void*)(p + m0 * ld), 0, __builtin_amdgcn_readfirstlane((int)(n * 2)), 0x00020000);
            };
            const __amdgpu_buffer_rsrc_t ry = resource(g.y, g.ldy), rr = resource(g.res, EPI == MX_RES ? g.ldr : 0);
            auto offset = [&](long ld, int m, int n, int t) { return c0 + n * 32 < g.N ? (int)((m * 32 + t * 16 + (lane & 15)) * ld + c0 + n * 32) * 2 : -16; };
            constexpr int POLICY = TM * TN < 8 ? WRITE_THROUGH : 0;  // (the large tile, 16384 x 640 x 5120: 56 us without, 61 with)
            constexpr int BLOCKS = TM * TN, AHEAD = BLOCKS < 5 ? BLOCKS : 5;  // (the residual of all blocks at once: registers for five)
            uint4v r[EPI == MX_RES ? BLOCKS : 1][2];
            auto residual = [&](int i) {
                if constexpr (EPI == MX_RES) {
#pragma unroll
                    for (int t = 0; t < 2; ++t) r[i][t] = __builtin_amdgcn_raw_buffer_load_b128(rr, offset(g.ldr, i / TN, i % TN, t), 0, 0);
                }
            };
#pragma unroll
            for (int i = 0; i < AHEAD; ++i) residual(i);
#pragma unroll
            for (int i = 0; i < BLOCKS; ++i) {
                uint4v v[2];
                mx_finish_block<DT>(acc[i / TN][i % TN], EPI == MX_RES ? r[EPI == MX_RES ? i : 0] : nullptr, v);
                if (i + AHEAD < BLOCKS) residual(i + AHEAD);  // (before the stores: waiting for it is not waiting for them)
#pragma unroll
                for (int t = 0; t < 2; ++t) __builtin_amdgcn_raw_buffer_store_b128(v[t], ry, offset(g.ldy, i / TN, i % TN, t), 0, POLICY);
            }
        } else {
#pragma unroll
            for (int n = 0; n < TN; ++n) {
                const int c = c0 + n * 32, left = g.N - c;
#pragma unroll
                for (int m = 0; m < TM; ++m) {
                    const long row = m0 + m * 32 + (lane & 15);
                    uint4v v[2], r[2] = {{0, 0, 0, 0}, {0, 0, 0, 0}};
                    if (g.res) {
#pragma unroll
                        for (int t = 0; t < 2; ++t)
                            if (row + 16 * t < g.M && left > 0) r[t] = load8_16(g.res + (row + 16 * t) * g.ldr + c, left);
                    }
                    mx_finish_block<DT>(acc[m][n], r, v);
#pragma unroll
                    for (int t = 0; t < 2; ++t)
                        if (row + 16 * t < g.M && left > 0) store8_16(g.y + (row + 16 * t) * g.ldy + c, v[t], left);
                }
            }
        }
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // (loads of no bytes still write their zeros)
}

template <int DT, int EPI, int WM, int WN, int TM, int TN, int S>
static int run_mx_form(const MxGemm& g, long band, long most, hipStream_t st) {
    using P = MxPlan<WM, WN, TM, TN, S>;
    const long rows = (g.a.groups + P::GA - 1) / P::GA, cols = (g.w.groups + P::GB - 1) / P::GB;
    auto kernel = mx_gemm_kernel<DT, EPI, WM, WN, TM, TN, S>;
    static PerDevice prepared;
    if (const int rc = allow_lds(prepared, (const void*)kernel, P::BYTES)) return rc;
    // (several tiles for a workgroup: where a tile has at least as many steps as there are slots)
    const long wgs = rows * cols <= most || (g.a.kc + 1) / 2 < S ? rows * cols : most;
    kernel<<<(unsigned)wgs, P::NW * 64, P::BYTES, st>>>(g, mx_tiles(rows, cols, band));
    MQ_HIP_CHECK_LAUNCH();
    return MQ_OK;
}

template <int DT, int WM, int WN, int TM, int TN, int S>
static int run_mx_gemm(const MxGemm& g, long band, long most, hipStream_t st) {
    auto wide = [](const void* p, long ld) { return (uintptr_t)p % 16 == 0 && ld % 8 == 0 && ld < (1 << 22); };  // (offsets of a tile are 32-bit)
    if (g.N % 8 != 0 || !wide(g.y, g.ldy) || (g.res && !wide(g.res, g.ldr)) || (uintptr_t)g.bias % 16 != 0)
        return run_mx_form<DT, MX_ODD, 2, 2, 2, 2, 4>(g, band, 1L << 31, st);
    return g.res ? run_mx_form<DT, MX_RES, WM, WN, TM, TN, S>(g, band, most, st) : run_mx_form<DT, MX_PLAIN, WM, WN, TM, TN, S>(g, band, most, st);
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

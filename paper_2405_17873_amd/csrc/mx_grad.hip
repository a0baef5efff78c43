// Gradient of a microscaled 4-bit linear with respect to its input: dX = dY W, the 4-bit weights widened to 16 bits on their way into the MFMAs.
//
// The reduction runs over the weights' rows n, along which neither codes nor scales are contiguous.  Widened 16-bit rows of k go to LDS and come back
// through the transposing LDS load, which hands a lane consecutive n of one column k.  In fp16, which has too few exponents for 2^(s - 127), widened
// weights are taken relative to the largest scale of their block column (top), and a value 2^-37 of its column's largest may go; the product is scaled
// back at the end, exactly.  bfloat16 has the exponents, and weights go in as they are: relative ones of ordinary layers were larger, and sums of a dY
// near the end of its range became infinite on the way to finite results.
#include "expert_walk.h"
#include "mx_common.h"

namespace mq {

typedef short short4v __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) short4v lds_short4v;
typedef __attribute__((address_space(3))) uint4v lds_uint4v;
typedef __attribute__((address_space(3))) uint32_t lds_uint;
typedef __attribute__((address_space(3))) float4v lds_float4v;

struct MxGrad {
    const uint16_t* dy;
    long lddy;
    MxView w;  // weights [N,K]
    const uint8_t* top;
    int M, N, K;
    uint16_t* dx;
    long lddx;
    bool wide;  // rows of dY start on 16-byte boundaries
    const int* offsets;  // by expert: w and top are the first expert's
    int experts;
};

// What is added to the scale bytes of a block column with the largest scale `top`, and taken back at the end.  fp16: 6 units of the largest are 49152.
// bfloat16: nothing, but that products of columns below 2^-60 keep clear of the subnormal floats, and that 6 units of the largest are a bfloat16 (beside
// scales past 252, which no quantiser makes, those of 0 and 1 count up to fourfold then; a mask of their codes costs 8192 x 8192 x 8192 1030 -> 1045 us).
template <int DT>
__device__ __forceinline__ int mx_grad_shift(int top) {
    return DT == MQ_F16 ? 140 - top : top < 64 ? 64 - top : top > 252 ? 252 - top : 0;
}
// Scale operand of a block with scale byte s.  (Exponent field 0 and below: nothing that fp16 holds.)
__device__ __forceinline__ float mx_grad_scale(uint32_t s, int shift) {
    const int f = (int)s + shift;
    return mx_scale_operand(s == 255u ? 255u : f > 0 ? (uint32_t)f : 0u);
}
template <int DT>
__device__ __forceinline__ uint4v mx_widen8(uint32_t w, float sc) {
    if constexpr (DT == MQ_F16)
        return uint4v{h2_bits(__builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, sc, 0)), h2_bits(__builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, sc, 1)),
                      h2_bits(__builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, sc, 2)), h2_bits(__builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, sc, 3))};
    else
        return uint4v{__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, sc, 0)),
                      __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, sc, 1)),
                      __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, sc, 2)),
                      __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, sc, 3))};
}
template <int DT>
__device__ __forceinline__ float16v mx_grad_mfma(uint4v w, uint4v d, float16v c) {
    if constexpr (DT == MQ_F16)
        return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(half8, w), __builtin_bit_cast(half8, d), c, 0, 0, 0);
    else
        return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, w), __builtin_bit_cast(bf16x8, d), c, 0, 0, 0);
}

// A tile of those that a walk has counted: it is at its last turn, which has the tile unless an earlier one does.
__device__ __forceinline__ MxPlanTile expert_tile(ExpertWalk& walk, const MxGrad& g, int number, int tile_rows) {
    if (number < walk.before) {
        walk = ExpertWalk{};
        for (;; walk.next()) {
            walk.load(g.offsets, g.experts, g.M, tile_rows, 0);
            if (number < walk.before + walk.turn_tiles) break;
        }
    }
    return walk.tile(number, tile_rows);
}

// Eight sums of a block column, scaled back and rounded.
template <int DT>
__device__ __forceinline__ uint4v mx_grad_result(float4v a, float4v b, int top) {
    const int back = -mx_grad_shift<DT>(top);
    return uint4v{T16<DT>::pack(ldexpf(a[0], back), ldexpf(a[1], back)), T16<DT>::pack(ldexpf(a[2], back), ldexpf(a[3], back)),
                  T16<DT>::pack(ldexpf(b[0], back), ldexpf(b[1], back)), T16<DT>::pack(ldexpf(b[2], back), ldexpf(b[3], back))};
}

// Work of one launch.  Whole rounds of tiles, one workgroup per compute unit, run undivided; the reduction of the `tiles - whole` that are left is cut into
// `parts`, whose sums go to the workspace and are joined by a second kernel.
struct GradWork {
    uint32_t col_tiles, whole, parts;
    float* partial;
};

// LDS-writing loads whose LDS address and scalar offset are sums: what has to lie between the address and the load is the other addition.
__device__ __forceinline__ void dma_step_b128(int4s rsrc, uint32_t lds_stage, uint32_t lds_offset, int voff, int soff, int soff2) {
    int sum;
    asm volatile("s_add_u32 m0, %1, %2\n\ts_add_u32 %0, %3, %4\n\tbuffer_load_dwordx4 %5, %6, %0 offen lds"
                 : "=&s"(sum)
                 : "s"(lds_stage), "s"(lds_offset), "s"(soff), "s"(soff2), "v"(voff), "s"(rsrc)
                 : "memory", "scc");
}
__device__ __forceinline__ void dma_step_b32(int4s rsrc, uint32_t lds_stage, uint32_t lds_offset, int voff, int soff) {
    asm volatile("s_add_u32 m0, %0, %1\n\ts_nop 0\n\tbuffer_load_dword %2, %3, %4 offen lds"
                 :
                 : "s"(lds_stage), "s"(lds_offset), "v"(voff), "s"(rsrc), "s"(soff)
                 : "memory", "scc");
}

// Rows of 64 bytes (or an odd number of them) in LDS: piece p of 16 bytes of row r lies at p ^ turned(r).  One piece of any 8 consecutive rows then lies in
// 8 different places of 128 bytes, and of 16 rows in 16 of 256.  (Against p ^ (r >> 2), which does the second alone: 8192 x 8192 x 8192 1130 -> 1080 us.)
__device__ __forceinline__ int mx_turned(int r) { return ((r >> 2) & 3) ^ (r & 2); }

// LDS plan of a workgroup of NW waves, each with all 32 TM x 128 results of the workgroup's tile and a share of the reduction.  A unit is the 32
// rows of one weight group: dY 32 TM rows x 32 n, the codes of four blocks, and their scale words.
template <int TM, int NW, int S>
struct GradPlan {
    static constexpr int TK = 4;  // blocks of 32 columns: a lane of a wave for each row (of 16) and block
    static constexpr int DY = TM * 2048, CODES = TK * 512, SCALES = 256, SLOT = DY + CODES + SCALES;
    static constexpr int DY_OPS = TM * 2, CODE_OPS = TK / 2, OPS = DY_OPS + CODE_OPS + 1;
    static constexpr int EARLY = OPS / 2;  // loads of a unit in the first half of another
    static constexpr int ROW = TK * 64 + 64;  // of widened weights: 16 words modulo the banks, so that four rows meet no conflict
    static constexpr int WAVE = S * SLOT + 16 * ROW;
    static constexpr int JROW = TK * 128 + 16, JOIN = 32 * JROW;  // one wave's 32 x 128 results on their way into the sum
    static constexpr int BYTES = NW * (WAVE > JOIN ? WAVE : JOIN);
};

// A wave has its own part of the reduction (units wv, wv + NW, ...) and its own LDS, and waits for nobody until the sums of the waves are joined: no
// weight is widened twice in a tile, and no operand is read from LDS by two waves.  128 x 128 results of a wave are what its registers hold; LDS holds
// three units then.
// Measured (bfloat16): 8192 x 8192 x 8192 1030 to 1045 us, 1.06 PFLOP/s (a library product of 16-bit matrices reaches 1.37), on zeros 870: a fifth is power.  With
// no loads from memory 790 us.  A unit (32 MFMAs, 1024 cycles) keeps LDS busy for about as long: loads write 41 KB, widened weights 32, reads fetch 73.
template <int DT, int TM, int NW, int S, bool EXPERTS>
__global__ __launch_bounds__(NW * 64, 1) void mx_grad_kernel(const MxGrad g, const GradWork work) {
    using P = GradPlan<TM, NW, S>;
    constexpr int TK = P::TK;
    extern __shared__ __attribute__((aligned(16))) uint8_t lds[];
    const int lane = threadIdx.x & 63, wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int h = lane >> 5;
    // whole tiles: neighbouring tiles of one row strip run on one XCD
    // (by expert, the launch has as many workgroups as there can be tiles, and each finds its own)
    ExpertWalk walk;
    if constexpr (EXPERTS) {
        for (;; walk.next()) {
            walk.load(g.offsets, g.experts, g.M, TM * 32, 0);
            if (walk.base + 64 >= g.experts) break;
        }
    }
    const uint32_t undivided = EXPERTS ? (uint32_t)(walk.before + walk.turn_tiles) * work.col_tiles : work.whole;
    const bool whole = EXPERTS || blockIdx.x < work.whole;
    const uint32_t xcd = blockIdx.x & 7, more = undivided & 7;
    if (EXPERTS && (blockIdx.x >> 3) >= (undivided >> 3) + (xcd < more ? 1u : 0u)) return;
    const uint32_t tile_v = whole ? xcd * (undivided >> 3) + (xcd < more ? xcd : more) + (blockIdx.x >> 3) : work.whole + (blockIdx.x - work.whole) / work.parts;
    const uint32_t tile = __builtin_amdgcn_readfirstlane(tile_v);  // (divisions are done in vector registers)
    const uint32_t part = whole ? 0 : (blockIdx.x - work.whole) % work.parts, parts = whole ? 1 : work.parts;
    const uint32_t tile_row = __builtin_amdgcn_readfirstlane(tile / work.col_tiles);
    long m0 = (long)tile_row * (TM * 32);
    int rows_end = g.M;
    const uint8_t *codes = g.w.codes, *scales = g.w.scales, *top = g.top;
    if constexpr (EXPERTS) {
        const MxPlanTile t = expert_tile(walk, g, (int)tile_row, TM * 32);
        m0 = t.start;
        rows_end = t.end;
        codes += (long)t.expert * g.w.groups * g.w.kc * 1024;
        scales += (long)t.expert * g.w.groups * g.w.kq * 256;
        top += (long)t.expert * (g.K >> 5);
    }
    const int b0 = __builtin_amdgcn_readfirstlane((int)(tile % work.col_tiles) * TK);  // first block column: half of a scale column
    const int kc = g.w.kc, kq = g.w.kq, blocks = g.K >> 5;
    const int g0 = __builtin_amdgcn_readfirstlane((int)((long)g.w.groups * part / parts)), g1 = __builtin_amdgcn_readfirstlane((int)((long)g.w.groups * (part + 1) / parts));
    const int units = (g1 - g0 - wv + NW - 1) / NW;  // of this wave; may be none
    const uint32_t base = (uint32_t)(uintptr_t)lds + wv * P::WAVE;
    constexpr int OOB = 0x7FFFF000;

    const long rows = rows_end - m0 < TM * 32 ? rows_end - m0 : TM * 32;
    const int n_end = g.N < g1 * 32 ? g.N : g1 * 32;
    const int4s rd = make_rsrc(g.dy + m0 * g.lddy, (uint32_t)(((rows - 1) * g.lddy + g.N) * 2));
    const int4s rc = make_rsrc(codes, (uint32_t)((long)g1 * kc * 1024));
    const int4s rs = make_rsrc(scales, (uint32_t)((long)g1 * kq * 256));
    // dY: a load takes 16 rows x 64 bytes; piece p of row r lies at p ^ turned(r)
    const int piece = (lane & 3) ^ mx_turned(lane >> 2);
    const int v_dy = (int)((long)(lane >> 2) * g.lddy * 2) + piece * 16;
    const int dy_step = (int)(g.lddy * 32);  // 16 rows
    // codes: a load takes the 32 rows of two blocks, a tile in lane order.  scales: the words of 32 rows x two blocks
    const int v_code = (b0 >> 1) * 1024 + lane * 16, v_scale = (b0 >> 3) * 256 + lane * 4;
    const bool second = b0 + 2 < blocks;

    uint32_t fill = 0;
    int ahead = 0, v_now = 0, s_dy = 0, s_code = 0, s_code2 = 0, s_scale = 0;
    auto load_unit = [&]() {  // sets up the loads of the wave's unit `ahead`; units past the end read as zero
        const bool live = ahead < units;
        const int grp = g0 + wv + ahead * NW;
        v_now = live && grp * 32 + piece * 8 < n_end ? v_dy : OOB;
        s_dy = __builtin_amdgcn_readfirstlane(grp * 64);
        s_code = __builtin_amdgcn_readfirstlane(live ? grp * kc * 1024 : OOB);
        s_code2 = __builtin_amdgcn_readfirstlane(live && second ? grp * kc * 1024 + 1024 : OOB);
        s_scale = __builtin_amdgcn_readfirstlane(live ? grp * kq * 256 : OOB);
        ++ahead;
    };
    auto load = [&](int i) {
        if (i < P::DY_OPS)
            dma_step_b128(rd, base + fill, i * 1024, v_now, s_dy, i * dy_step);
        else if (i < P::DY_OPS + P::CODE_OPS)
            dma_step_b128(rc, base + fill, P::DY + (i - P::DY_OPS) * 1024, v_code, i == P::DY_OPS ? s_code : s_code2, 0);
        else
            dma_step_b32(rs, base + fill, P::DY + P::CODES, v_scale, s_scale);
    };
    auto load_done = [&]() { fill = fill == (S - 1) * P::SLOT ? 0 : fill + P::SLOT; };

    // widening: the lane has row wn (of 16) of block wb; its four pieces of eight columns lie at p ^ turned(wn)
    const int wn = lane & 15, wb = lane >> 4;
    const int b_mine = b0 + wb < blocks ? b0 + wb : blocks - 1;
    const int shift = mx_grad_shift<DT>((int)top[b_mine]), sbit = 8 * ((b_mine >> 1) & 3);
    const uint32_t a_code = base + P::DY + wb * 512 + wn * 16, a_scale = base + P::DY + P::CODES + (b_mine & 1) * 128 + wn * 4;
    const uint32_t a_wide = base + S * P::SLOT;
    uint32_t a_write[4], a_read[2];
#pragma unroll
    for (int i = 0; i < 4; ++i) a_write[i] = a_wide + wn * P::ROW + wb * 64 + ((i ^ mx_turned(wn)) << 4);
#pragma unroll
    for (int u = 0; u < 2; ++u) {  // 16 lanes read 4 rows of 16 columns and get 4 rows of their column
        const int n = h * 8 + u * 4 + ((lane & 15) >> 2);
        a_read[u] = a_wide + n * P::ROW + (((((lane >> 4) & 1) * 2 + ((lane & 3) >> 1)) ^ mx_turned(n)) << 4) + (lane & 1) * 8;
    }
    const int r = lane & 31;
    uint32_t a_dy[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) a_dy[i] = base + r * 64 + (((i * 2 + h) ^ mx_turned(r)) << 4);

    struct Frag {
        uint4v w[TK], d[TM];
    } f0, f1;
    uint4v code = {0, 0, 0, 0};
    uint32_t word = 0, at_dy = 0;
    float scale = 0.0f;
    // On the way to the fragments of k step s (16 n) of the unit in `slot`, in this order: one read of codes and scales, TM reads of dY, four writes of
    // widened weights, TK reads of them.
    auto prepare = [&](Frag& f, uint32_t slot, int s, int i) {
        if (i == 0) {
            code = *(const lds_uint4v*)(uintptr_t)(a_code + slot + s * 256);
            word = *(const lds_uint*)(uintptr_t)(a_scale + slot + s * 64);
            at_dy = a_dy[s] + slot;
        } else if (i < 1 + TM) {
            const int j = i - 1;
            f.d[j < TM ? j : 0] = ((const lds_uint4v*)(uintptr_t)at_dy)[j * 128];
        } else if (i < 5 + TM) {
            const int j = i - 1 - TM;
            if (j == 0) scale = mx_grad_scale((word >> sbit) & 255u, shift);
            *(lds_uint4v*)(uintptr_t)a_write[j & 3] = mx_widen8<DT>(code[j & 3], scale);
        } else {
            const int j = i - 5 - TM;
            const uint2v lo = __builtin_bit_cast(uint2v, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_short4v*)(uintptr_t)(a_read[0]) + j * 8));
            const uint2v hi = __builtin_bit_cast(uint2v, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_short4v*)(uintptr_t)(a_read[1]) + j * 8));
            f.w[j < TK ? j : 0] = uint4v{lo[0], lo[1], hi[0], hi[1]};
        }
    };
    constexpr int PREPARE = 5 + TM + TK;

    float16v acc[TM][TK];
    // The MFMAs of a k step, and between them the way to the next fragments, which ends three quarters through so that nobody waits for them, and
    // the loads first .. last - 1.
    auto phase = [&](const Frag& f, Frag& next, uint32_t slot, int s, int first, int last) {
        constexpr int MM = TM * TK, SPAN = MM * 7 / 8;
#pragma unroll
        for (int i = 0; i < MM; ++i) {
            const int m = i % TM, k = i / TM;  // (weights, which are ready last, one after the other)
            acc[m][k] = mx_grad_mfma<DT>(f.w[k], f.d[m], acc[m][k]);
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int j = i * PREPARE / SPAN; j < (i + 1) * PREPARE / SPAN && j < PREPARE; ++j) prepare(next, slot, s, j);
#pragma unroll
            for (int j = i * (last - first) / MM; j < (i + 1) * (last - first) / MM; ++j) load(first + j);
            __builtin_amdgcn_sched_barrier(0);
        }
    };

#pragma unroll
    for (int u = 0; u < S - 1; ++u) {
        load_unit();
#pragma unroll
        for (int i = 0; i < P::OPS; ++i) load(i);
        load_done();
    }
#pragma unroll
    for (int m = 0; m < TM; ++m)
#pragma unroll
        for (int k = 0; k < TK; ++k)
#pragma unroll
            for (int i = 0; i < 16; ++i) acc[m][k][i] = 0.0f;
    wait_vmcnt<(S - 2) * P::OPS>();
#pragma unroll
    for (int i = 0; i < PREPARE; ++i) prepare(f0, 0, 0, i);
    uint32_t slot = 0;
    for (int u = 0; u < units; ++u) {
        load_unit();
        phase(f0, f1, slot, 1, 0, P::EARLY);  // (the unit before is read out: its last fragments have been multiplied)
        slot = slot == (S - 1) * P::SLOT ? 0 : slot + P::SLOT;
        wait_vmcnt<(S - 3) * P::OPS + P::EARLY>();
        phase(f1, f0, slot, 0, P::EARLY, P::OPS);
        load_done();
    }
    wait_vmcnt<0>();
    __syncthreads();

    // The waves' sums, 32 rows at a time: each wave puts its own into LDS, all threads add them up in wave order.
    constexpr int VECS = 32 * TK * 4, PER = (VECS + NW * 64 - 1) / (NW * 64);  // runs of eight columns
    const uint32_t join = (uint32_t)(uintptr_t)lds;
#pragma unroll
    for (int m = 0; m < TM; ++m) {
        if (m0 + m * 32 >= rows_end) break;
        if (m) __syncthreads();
#pragma unroll
        for (int k = 0; k < TK; ++k)
#pragma unroll
            for (int t = 0; t < 4; ++t)
                *(lds_float4v*)(uintptr_t)(join + wv * P::JOIN + r * P::JROW + k * 128 + t * 32 + h * 16) =
                    float4v{acc[m][k][4 * t], acc[m][k][4 * t + 1], acc[m][k][4 * t + 2], acc[m][k][4 * t + 3]};
        __syncthreads();
#pragma unroll
        for (int p = 0; p < PER; ++p) {
            const int v = p * NW * 64 + (int)threadIdx.x;
            const int row = v / (TK * 4), c = v % (TK * 4);
            const long mm = m0 + m * 32 + row;
            const int k = b0 * 32 + c * 8;
            if (v < VECS && mm < rows_end && k < g.K) {
                float4v a = {0, 0, 0, 0}, b = {0, 0, 0, 0};
#pragma unroll
                for (int w = 0; w < NW; ++w) {
                    const uint32_t at = join + w * P::JOIN + row * P::JROW + c * 32;
                    a += *(const lds_float4v*)(uintptr_t)at;
                    b += *(const lds_float4v*)(uintptr_t)(at + 16);
                }
                if (whole) {
                    store8_16(g.dx + mm * g.lddx + k, mx_grad_result<DT>(a, b, (int)top[k >> 5]), 8);
                } else {
                    float* out = work.partial + ((long)(blockIdx.x - work.whole) * (TM * 32) + m * 32 + row) * (TK * 32) + c * 8;
                    *(float4v*)out = a;
                    *(float4v*)(out + 4) = b;
                }
            }
        }
    }
}

// Adds up the parts of the tiles whose reduction was cut, in order: a thread for eight columns of a row.
template <int DT>
__global__ __launch_bounds__(256) void mx_grad_join_kernel(const MxGrad g, const GradWork work, const int tile_rows, const uint32_t tiles) {
    const uint32_t v = blockIdx.x * 256 + threadIdx.x;
    const uint32_t c = v & 15, row = (v >> 4) % tile_rows, t = (v >> 4) / tile_rows, tile = work.whole + t;
    if (tile >= tiles) return;
    const long m = (long)(tile / work.col_tiles) * tile_rows + row;
    const int k = (int)(tile % work.col_tiles) * 128 + (int)c * 8;
    if (m >= g.M || k >= g.K) return;
    const float* p = work.partial + ((long)t * work.parts * tile_rows + row) * 128 + c * 8;
    float4v a = *(const float4v*)p, b = *(const float4v*)(p + 4);
    for (uint32_t i = 1; i < work.parts; ++i) {
        p += (long)tile_rows * 128;
        a += *(const float4v*)p;
        b += *(const float4v*)(p + 4);
    }
    store8_16(g.dx + m * g.lddx + k, mx_grad_result<DT>(a, b, (int)g.top[k >> 5]), 8);
}

// Any alignment of dY's rows, any N, weights of any size: 64 x 64 results per workgroup, operands through registers.
template <int DT, bool EXPERTS>
__global__ __launch_bounds__(256) void mx_grad_any_kernel(const MxGrad g) {
    constexpr int BM = 64, BK = 64, BN = 64;
    __shared__ __attribute__((aligned(16))) uint8_t wt[BN * BK * 2];
    __shared__ __attribute__((aligned(16))) uint8_t dt[BM * BN * 2];
    const int tid = threadIdx.x, lane = tid & 63, wv = __builtin_amdgcn_readfirstlane(tid >> 6);
    long m0 = (long)blockIdx.x * BM;
    int rows_end = g.M;
    const uint8_t *codes = g.w.codes, *scales = g.w.scales, *top = g.top;
    if constexpr (EXPERTS) {
        ExpertWalk walk;
        for (;; walk.next()) {
            walk.load(g.offsets, g.experts, g.M, BM, 0);
            if ((int)blockIdx.x < walk.before + walk.turn_tiles) break;
            if (walk.base + 64 >= g.experts) return;
        }
        const MxPlanTile t = walk.tile((int)blockIdx.x, BM);
        m0 = t.start;
        rows_end = t.end;
        codes += (long)t.expert * g.w.groups * g.w.kc * 1024;
        scales += (long)t.expert * g.w.groups * g.w.kq * 256;
        top += (long)t.expert * (g.K >> 5);
    }
    const int c = blockIdx.y, k0 = c * BK;
    const int wm = wv & 1, wk = wv >> 1;
    float16v acc = {};
    for (int n0 = 0; n0 < g.N; n0 += BN) {
        __syncthreads();
        if (tid < 128) {
            const int grp = tid >> 6, L = tid & 63, j = L & 31, kb = L >> 5, n = grp * 32 + j;
            uint4v v = {0, 0, 0, 0};
            uint32_t s = 0, t = 0;
            if (n0 / 32 + grp < g.w.groups) {
                const long G = n0 / 32 + grp;
                v = *(const uint4v*)(codes + (G * g.w.kc + c) * 1024 + L * 16);
                s = scales[(G * g.w.kq + (c >> 2)) * 256 + L * 4 + (c & 3)];
                const int b = c * 2 + kb;
                t = b * 32 < g.K ? top[b] : 0;
            }
            const float sc = mx_grad_scale(s, mx_grad_shift<DT>((int)t));
#pragma unroll
            for (int i = 0; i < 4; ++i) *(uint4v*)(wt + n * (BK * 2) + (((kb * 4 + i) ^ (n & 7)) << 4)) = mx_widen8<DT>(v[i], sc);
        }
#pragma unroll
        for (int i = 0; i < 2; ++i) {  // dY: 64 rows of 8 pieces
            const int t = i * 256 + tid, r = t >> 3, p = t & 7;
            const int n = n0 + p * 8;
            uint4v v = {0, 0, 0, 0};
            if (m0 + r < rows_end && n < g.N) v = load8_16(g.dy + (m0 + r) * g.lddy + n, g.N - n);
            *(uint4v*)(dt + r * (BN * 2) + ((p ^ (r & 7)) << 4)) = v;
        }
        __syncthreads();
#pragma unroll
        for (int s = 0; s < 4; ++s) {
            const int h = lane >> 5;
            const int r = wm * 32 + (lane & 31), p = s * 2 + h;
            const uint4v b = *(const uint4v*)(dt + r * (BN * 2) + ((p ^ (r & 7)) << 4));
            uint2v a[2];
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                const int n = s * 16 + h * 8 + u * 4 + ((lane & 15) >> 2);
                const int col = wk * 32 + ((lane >> 4) & 1) * 16 + (lane & 3) * 4;
                const uint32_t at = (uint32_t)(uintptr_t)wt + (uint32_t)(n * (BK * 2) + (((col >> 3) ^ (n & 7)) << 4) + (col & 4) * 2);
                a[u] = __builtin_bit_cast(uint2v, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_short4v*)(uintptr_t)at));
            }
            acc = mx_grad_mfma<DT>(uint4v{a[0][0], a[0][1], a[1][0], a[1][1]}, b, acc);
        }
    }
    const long m = m0 + wm * 32 + (lane & 31);
    const int kcol = k0 + wk * 32, h = lane >> 5;
    if (kcol >= g.K || m >= rows_end) return;
    const int back = -mx_grad_shift<DT>((int)top[kcol >> 5]);
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        const int k = kcol + 8 * (i >> 2) + 4 * h + (i & 3);
        g.dx[m * g.lddx + k] = T16<DT>::down(ldexpf(acc[i], back));
    }
}

// Rows of dY that do not start on 16-byte boundaries, or end inside a vector of eight, copied to rows that do neither; what is past their end is zero.
// A wave takes 256 vectors of a row.
__global__ __launch_bounds__(256) void mx_grad_align_kernel(const uint16_t* dy, long lddy, int M, int N, uint16_t* to, int ld) {
    const long m = blockIdx.x * 4L + (threadIdx.x >> 6);
    const int n0 = (int)blockIdx.y * 2048 + (threadIdx.x & 63) * 8;
    if (m >= M) return;
    uint4v v[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = n0 + i * 512 < N ? load8_16(dy + m * lddy + n0 + i * 512, N - n0 - i * 512) : uint4v{0, 0, 0, 0};
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (n0 + i * 512 < N) *(uint4v*)(to + m * ld + n0 + i * 512) = v[i];
}

// The form for a problem: 32, 64 or 128 rows of a tile, and how the last round of tiles is cut, by what it is estimated to take: a launch, and for every
// round of 256 workgroups a fixed part (filling the pipeline, joining the waves) and one per unit of a wave.  us, estimate (measured) for 32 / 64 / 128
// rows: 308 x 2048 x 640 8.6 (7.5) / 9.9 (9.0) / 11.9 (11.7), 1000 x 992 x 1000 9.6 (9.1) / 11.9 (10.9) / 15 (14), 4096 x 1280 x 1280 43 (43) / 35 (35) /
// 32 (32), 8 x 5120 x 20480 in six parts 22 (22) / 27 (26) / 37 (35).
struct GradForm {
    int tm;
    long tiles, whole, parts;
    double us;
};
static GradForm mx_grad_form(long M, long N, long K, int tm, int waves, double per_unit, double per_round) {
    GradForm f;
    f.tm = tm;
    f.tiles = (M + tm * 32 - 1) / (tm * 32) * ((K / 32 + 3) / 4);
    f.whole = f.tiles / 256 * 256;
    const long left = f.tiles - f.whole, units = ((N + 31) / 32 + waves - 1) / waves;  // of a wave
    f.parts = 1;
    if (left > 0) {
        f.parts = 256 / left < units / 8 ? 256 / left : units / 8;
        if (f.parts < 1) f.parts = 1;
    }
    if (f.parts == 1) f.whole = f.tiles;
    const double rounds = (double)((f.whole + 255) / 256);
    f.us = 2.5 + rounds * (units * per_unit + per_round);
    if (f.parts > 1) f.us += units * per_unit / f.parts + per_round + 3.0;
    return f;
}
static GradForm mx_grad_form(long M, long N, long K) {
    const GradForm f[3] = {mx_grad_form(M, N, K, 1, 8, 0.97, 3.2), mx_grad_form(M, N, K, 2, 4, 0.68, 4.0), mx_grad_form(M, N, K, 4, 4, 1.04, 4.2)};
    const int i = f[1].us < f[0].us ? 1 : 0;
    return f[2].us < f[i].us ? f[2] : f[i];
}
static size_t mx_grad_partial_bytes(long M, long N, long K) {
    const GradForm f = mx_grad_form(M, N, K);
    return f.parts > 1 ? (size_t)(f.tiles - f.whole) * f.parts * f.tm * 32 * 128 * 4 : 0;
}
// Whether dY is copied to aligned rows, for the sake of long reductions.  us, copied / any alignment: 11060 x 384 x 8716 171 / 240, 1 x 384 x 10519 16 / 110,
// 2000 x 4000 x 2001 52 / 91, 2 x 7840 x 655 9.5 / 9.8, 3000 x 1280 x 515 17.2 / 17.7; 5000 x 320 x 260 12 / 8.5, 16384 x 640 x 100 31 / 16, 16 x 1280 x 33 7.5 / 3.5
// (and 4096 x 1280 x 1283 41 / 37).
static bool mx_grad_copies(long N) { return N % 8 != 0 && N > 512; }
size_t mx_grad_workspace_bytes(long M, long N, long K) {
    return up256(mx_grad_partial_bytes(M, N, K)) + (mx_grad_copies(N) ? (size_t)M * ((N + 7) / 8 * 8) * 2 : 0);
}

template <int DT, int TM, int NW, int S>
static int run_mx_grad(const MxGrad& g, const GradForm& f, float* ws, hipStream_t st) {
    using P = GradPlan<TM, NW, S>;
    static_assert(P::BYTES <= 160 * 1024, "LDS of a compute unit");
    auto kernel = mx_grad_kernel<DT, TM, NW, S, false>;
    static PerDevice prepared;
    if (const int rc = allow_lds(prepared, (const void*)kernel, P::BYTES)) return rc;
    GradWork w;
    w.col_tiles = (uint32_t)((g.K / 32 + 3) / 4);
    w.whole = (uint32_t)f.whole;
    w.parts = (uint32_t)f.parts;
    w.partial = ws;
    const long left = f.tiles - f.whole;
    kernel<<<(unsigned)(f.whole + left * f.parts), NW * 64, P::BYTES, st>>>(g, w);
    MQ_HIP_CHECK_LAUNCH();
    if (left > 0) {
        mx_grad_join_kernel<DT><<<(unsigned)((left * TM * 32 * 16 + 255) / 256), 256, 0, st>>>(g, w, TM * 32, (uint32_t)f.tiles);
        MQ_HIP_CHECK_LAUNCH();
    }
    return MQ_OK;
}

template <int DT>
static int choose_mx_grad(MxGrad g, float* ws, hipStream_t st) {
    // 32-bit offsets of the loads: a row strip of dY, the weights' codes
    const bool small = (long)g.w.groups * g.w.kc * 1024 < (1L << 31);
    if (small && mx_grad_copies(g.N)) {
        const int ld = (g.N + 7) / 8 * 8;
        uint16_t* to = (uint16_t*)((char*)ws + up256(mx_grad_partial_bytes(g.M, g.N, g.K)));
        mx_grad_align_kernel<<<dim3((unsigned)((g.M + 3L) / 4), (unsigned)((g.N + 2047) / 2048)), 256, 0, st>>>(g.dy, g.lddy, g.M, g.N, to, ld);
        MQ_HIP_CHECK_LAUNCH();
        g.dy = to, g.lddy = g.N = ld, g.wide = true;
    }
    if (!g.wide || g.N % 8 != 0 || !small || g.lddy >= (1 << 22)) {
        mx_grad_any_kernel<DT, false><<<dim3((unsigned)((g.M + 63L) / 64), (unsigned)g.w.kc), 256, 0, st>>>(g);
        MQ_HIP_CHECK_LAUNCH();
        return MQ_OK;
    }
    const GradForm f = mx_grad_form(g.M, g.N, g.K);
    return f.tm == 1 ? run_mx_grad<DT, 1, 8, 3>(g, f, ws, st) : f.tm == 2 ? run_mx_grad<DT, 2, 4, 5>(g, f, ws, st) : run_mx_grad<DT, 4, 4, 3>(g, f, ws, st);
}

int launch_mx_grad(const void* dy, int M, int N, long lddy, const void* w, const uint8_t* top, int K, void* dx, long lddx, int dtype, void* ws,
                   hipStream_t st) {
    MxGrad g = {};
    g.dy = (const uint16_t*)dy;
    g.lddy = M > 1 ? lddy : N;
    g.w = mx_view(w, N, K);
    g.top = top;
    g.M = M;
    g.N = N;
    g.K = K;
    g.dx = (uint16_t*)dx;
    g.lddx = lddx;
    g.wide = (M == 1 || g.lddy % 8 == 0) && (uintptr_t)dy % 16 == 0;
    return dtype == MQ_F16 ? choose_mx_grad<MQ_F16>(g, (float*)ws, st) : choose_mx_grad<MQ_BF16>(g, (float*)ws, st);
}

// By expert: row tiles that start at the experts' first rows, and a workgroup for every tile that there can be.  Tiles of 32, 64 or 128 rows by the average number
// of an expert's rows.  us (bfloat16), 32 / 64 / 128: 1024 rows of 32 experts, 2048 x 2560, 41 / 47 / 43, 2048 76 / 52 / 62, 4096 122 / 93 / 69; 512 rows of 16, 1280 x 2048,
// 13.8 / 15.8 / 19.3, 1024 23.6 / 16.4 / 20.6, 2048 34.5 / 29.3 / 21.7; 512 of 64, 1280 x 1280, 26.5 / 29.0 / 36.1.  4001 rows of 16, 1280 x 2048, 39 to 43: some 390 tiles of 128 rows
// on 256 compute units are two rounds.
template <int DT, int TM, int NW, int S>
static int run_mx_experts_grad(const MxGrad& g, hipStream_t st) {
    using P = GradPlan<TM, NW, S>;
    auto kernel = mx_grad_kernel<DT, TM, NW, S, true>;
    static PerDevice prepared;
    if (const int rc = allow_lds(prepared, (const void*)kernel, P::BYTES)) return rc;
    GradWork w = {};
    w.col_tiles = (uint32_t)((g.K / 32 + 3) / 4);
    w.parts = 1;
    kernel<<<(unsigned)((mx_plan_bound(g.M, g.experts, TM * 32) * w.col_tiles + 7) / 8 * 8), NW * 64, P::BYTES, st>>>(g, w);
    MQ_HIP_CHECK_LAUNCH();
    return MQ_OK;
}
template <int DT>
static int choose_mx_experts_grad(const MxGrad& g, hipStream_t st) {
    if (!g.wide || g.lddy >= (1 << 22) || (long)g.w.groups * g.w.kc * 1024 >= (1L << 31)) {
        mx_grad_any_kernel<DT, true><<<dim3((unsigned)mx_plan_bound(g.M, g.experts, 64), (unsigned)g.w.kc), 256, 0, st>>>(g);
        MQ_HIP_CHECK_LAUNCH();
        return MQ_OK;
    }
    return g.M <= 32L * g.experts ? run_mx_experts_grad<DT, 1, 8, 3>(g, st) : g.M <= 64L * g.experts ? run_mx_experts_grad<DT, 2, 4, 5>(g, st) : run_mx_experts_grad<DT, 4, 4, 3>(g, st);
}
int launch_mx_experts_grad(const void* dy, int M, int N, long lddy, const void* w, const uint8_t* top, int K, int experts, const int* offsets, void* dx, long lddx,
                           int dtype, hipStream_t st) {
    MxGrad g = {};
    g.dy = (const uint16_t*)dy;
    g.lddy = M > 1 ? lddy : N;
    g.w = mx_view(w, N, K);
    g.w.scales = g.w.codes + (size_t)experts * g.w.groups * g.w.kc * 1024;
    g.top = top;
    g.M = M;
    g.N = N;
    g.K = K;
    g.dx = (uint16_t*)dx;
    g.lddx = lddx;
    g.wide = (M == 1 || g.lddy % 8 == 0) && (uintptr_t)dy % 16 == 0;
    g.offsets = offsets;
    g.experts = experts;
    return dtype == MQ_F16 ? choose_mx_experts_grad<MQ_F16>(g, st) : choose_mx_experts_grad<MQ_BF16>(g, st);
}

}  // namespace mq

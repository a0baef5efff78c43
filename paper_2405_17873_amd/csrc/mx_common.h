// Microscaled 4-bit floats (MXFP4): layout in memory, conversion, and what the kernels on them share.
//
// Every 32 consecutive values of a row form a block: 32 e2m1 codes (sign, 0 / 0.5 / 1 / 1.5 / 2 / 3 / 4 / 6) and one scale byte s that stands
// for 2^(s - 127), 255 for NaN.  s = max(0, E - 2) with E the biased binary32 exponent of the block's largest magnitude (the power of two
// below it is 4 units of the code, the largest binade of e2m1), 255 if the block holds an infinity or a NaN; codes round to nearest, ties to
// the even code, and magnitudes past 6 units become 6.
//
// In memory the unit is the block's 16 bytes of codes (code 2i in the low half of byte i), and blocks lie in the order in which a 32x32x64
// MFMA wants them: lane L = kb * 32 + j of a wave owns block kb (of two) of row j (of 32).
//   codes   tile (g, c), rows 32 g .. 32 g + 31, columns 64 c .. 64 c + 63: 1024 bytes at (g * KC + c) * 1024, lane L's block at 16 L;
//   scales  behind the codes, 256 bytes for four tiles (g, 4 q .. 4 q + 3) at (g * KQ + q) * 256: a word at 4 L, byte i for tile 4 q + i.
// A wave so fetches an operand with one contiguous load, and the scales of four operands with another; one word feeds four MFMAs, which pick
// their byte of it.  Rows are padded to 32, columns to 64 (scales to 256): padding holds code 0, scale 0, and so adds nothing to a product.
#pragma once
#include "gemm_core.h"
#include "per_device.h"

namespace mq {

struct MxView {  // host and device: where the parts of a matrix of `rows` x K lie
    const uint8_t* codes;
    const uint8_t* scales;
    int groups, kc, kq;
};
inline size_t mx_bytes(long rows, long K) {
    const size_t G = (size_t)(rows + 31) / 32, KC = (size_t)(K + 63) / 64, KQ = (KC + 3) / 4;
    return G * KC * 1024 + G * KQ * 256;
}
inline MxView mx_view(const void* p, long rows, long K) {
    MxView v;
    v.groups = (int)((rows + 31) / 32);
    v.kc = (int)((K + 63) / 64);
    v.kq = (v.kc + 3) / 4;
    v.codes = (const uint8_t*)p;
    v.scales = v.codes + (size_t)v.groups * v.kc * 1024;
    return v;
}

// 16-bit types by their dtype number.
template <int DT>
struct T16;
template <>
struct T16<MQ_F16> {
    static __device__ __forceinline__ float up(uint16_t b) { return (float)__builtin_bit_cast(_Float16, b); }
    static __device__ __forceinline__ uint16_t down(float f) { return __builtin_bit_cast(uint16_t, (_Float16)f); }
    static __device__ __forceinline__ uint32_t pack(float a, float b) {
        typedef float floats __attribute__((ext_vector_type(2)));
        typedef _Float16 halves __attribute__((ext_vector_type(2)));
        return __builtin_bit_cast(uint32_t, __builtin_convertvector((floats{a, b}), halves));  // (one instruction, to nearest)
    }
};
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
// (By value: the compiler reads element 0 where an element of a vector is bit-cast in place.)
__device__ __forceinline__ bf16x2 as_bf2(uint32_t u) { return __builtin_bit_cast(bf16x2, u); }
template <>
struct T16<MQ_BF16> {
    static __device__ __forceinline__ float up(uint16_t b) { return bf16_bits_to_float(b); }
    static __device__ __forceinline__ uint16_t down(float f) { return float_to_bf16_bits(f); }
    static __device__ __forceinline__ uint32_t pack(float a, float b) { return __builtin_bit_cast(uint32_t, bf16x2{(__bf16)a, (__bf16)b}); }
};

// Scale byte of a block from the bits of its largest magnitude (binary32, sign cleared; compared as integers, so that a NaN wins).
__device__ __forceinline__ uint32_t mx_scale_byte(uint32_t top_bits) {
    const uint32_t e = top_bits >> 23;
    return e == 255u ? 255u : e > 2u ? e - 2u : 0u;
}
// The conversion instructions take the scale as the exponent field of a float (field 0 stands for 2^-127, as in the byte).
__device__ __forceinline__ float mx_scale_operand(uint32_t byte) { return __uint_as_float(byte << 23); }

// Eight values -> eight codes.
template <int DT>
__device__ __forceinline__ uint32_t mx_codes_16(uint4v v, float scale) {
    uint32_t w = 0;
    if constexpr (DT == MQ_F16) {
        w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(w, as_h2(v[0]), scale, 0);
        w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(w, as_h2(v[1]), scale, 1);
        w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(w, as_h2(v[2]), scale, 2);
        w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(w, as_h2(v[3]), scale, 3);
    } else {
        w = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, as_bf2(v[0]), scale, 0);
        w = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, as_bf2(v[1]), scale, 1);
        w = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, as_bf2(v[2]), scale, 2);
        w = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, as_bf2(v[3]), scale, 3);
    }
    return w;
}
__device__ __forceinline__ uint32_t mx_codes_f32(const float* f, float scale) {
    uint32_t w = 0;
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, f[0], f[1], scale, 0);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, f[2], f[3], scale, 1);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, f[4], f[5], scale, 2);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, f[6], f[7], scale, 3);
    return w;
}

typedef uint16_t ushort2v __attribute__((ext_vector_type(2)));
// Largest of eight 16-bit magnitudes, as the bits of a binary32.
template <int DT>
__device__ __forceinline__ uint32_t mx_top_16(uint4v v) {
    ushort2v m = __builtin_bit_cast(ushort2v, v[0] & 0x7FFF7FFFu);
#pragma unroll
    for (int i = 1; i < 4; ++i) m = __builtin_elementwise_max(m, __builtin_bit_cast(ushort2v, v[i] & 0x7FFF7FFFu));
    const uint16_t t = m[0] > m[1] ? m[0] : m[1];
    return __float_as_uint(T16<DT>::up(t));
}

// Maximum over the four lanes (aligned) that share a block.
__device__ __forceinline__ uint32_t quad_max(uint32_t v) {
    uint32_t o = (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0xB1, 0xF, 0xF, true);  // lanes 1,0,3,2
    v = v > o ? v : o;
    o = (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0x4E, 0xF, 0xF, true);  // lanes 2,3,0,1
    return v > o ? v : o;
}

// Cache policy of buffer stores: through to memory at once, rather than when the kernel ends and waits for its caches to be written back.  4096 x 1280 x
// 1280 with a residual 12.5 to 11.3 us, 2964 x 1280 x 3840 16.9 to 13.9, the norm's backward pass over 16384 x 640 two of 30.
constexpr int WRITE_THROUGH = 17;

// Eight consecutive 16-bit values of a row, of which the first `n` exist (n >= 8: all), wherever they start: the memory takes 16 bytes at any address.
typedef uint4v uint4v_any __attribute__((aligned(2)));
__device__ __forceinline__ uint4v load8_16(const uint16_t* p, int n) {
    uint4v r = {0, 0, 0, 0};
    if (n >= 8) return *(const uint4v_any*)p;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t lo = 2 * i < n ? p[2 * i] : 0, hi = 2 * i + 1 < n ? p[2 * i + 1] : 0;
        r[i] = lo | hi << 16;
    }
    return r;
}
__device__ __forceinline__ void store8_16(uint16_t* p, uint4v v, int n) {
    if (n >= 8) {
        *(uint4v_any*)p = v;
        return;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if (2 * i < n) p[2 * i] = (uint16_t)v[i];
        if (2 * i + 1 < n) p[2 * i + 1] = (uint16_t)(v[i] >> 16);
    }
}

// Quantisation to MXFP4 by a workgroup of 256 threads: rows 32 g .. 32 g + 31, columns 256 q .. 256 q + 255.
// A lane converts eight consecutive values; four lanes share a block, and a wave covers 8 rows x 64 columns at a time, so that it reads
// whole 128-byte pieces of eight rows and writes two of 128 bytes (8 neighbouring rows of one block column).  Four such steps, 256 columns, make the
// scale word of a row and block column.  Bound by memory: 2 bytes read and 17/32 written per value.
template <int DT>
__device__ __forceinline__ void mx_quantize_groups(const uint16_t* x, int M, int K, long ldx, uint8_t* codes, uint8_t* scales, int kc, int kq, long g, int q) {
    const int lane = threadIdx.x & 63, sub = threadIdx.x >> 6;  // (a wave takes eight of the rows)
    if (g * 32 >= M) return;
    const int j = sub * 8 + (lane >> 3), kb = (lane >> 2) & 1, part = lane & 3;
    const long row = g * 32 + j;
    const int k0 = q * 256 + (lane & 7) * 8;
    const uint16_t* p = x + row * ldx + k0;
    uint4v v[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const bool in = row < M && k0 + 64 * i < K;  // K % 32 == 0: a block is whole or absent
        v[i] = in ? load8_16(p + 64 * i, 8) : uint4v{0, 0, 0, 0};
    }
    uint32_t word = 0;
    uint8_t* tile = codes + (g * kc + q * 4) * 1024 + (kb * 32 + j) * 16 + part * 4;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t s = mx_scale_byte(quad_max(mx_top_16<DT>(v[i])));
        uint32_t w = mx_codes_16<DT>(v[i], mx_scale_operand(s));
        if (s == 255u) w = 0;
        word |= s << (8 * i);
        if (q * 4 + i < kc) *(uint32_t*)(tile + (long)i * 1024) = w;
    }
    if (part == 0) *(uint32_t*)(scales + (g * kq + q) * 256 + (kb * 32 + j) * 4) = word;
}

inline size_t up256(size_t v) { return (v + 255) / 256 * 256; }

// Allows a kernel more than 64 KB of dynamic LDS on the current device.  `prepared`: the kernel's own.
inline int allow_lds(PerDevice& prepared, const void* kernel, int bytes) {
    int device = -1;
    if (hipGetDevice(&device) != hipSuccess) device = -1;
    return prepared(device, [&]() -> int {
        if (hipFuncSetAttribute(kernel, hipFuncAttributeMaxDynamicSharedMemorySize, bytes) == hipSuccess) return MQ_OK;
        set_hip_error((int)hipGetLastError());
        return MQ_ERR_HIP;
    });
}

// What else a kernel of the product does: an activation on the sums (g.act, which may be none), and the sums themselves to g.pre if asked for; a gate: the columns of Y are
// half those of the weights, the first half's sums times the activation of the second's; rows sorted by expert, the tiles by a plan made on the GPU.
enum { MX_ACT = 1, MX_GATED = 2, MX_EXPERTS = 4 };

// ---- launchers (arguments are checked by the entry points) ----
struct MxGemm {
    MxView a, w;  // activations [M,K], weights [N,K]
    int M, N, K;
    const uint16_t* bias;
    uint16_t* y;
    long ldy;
    const uint16_t* res;
    long ldr;
    int dtype;
    // with an activation
    int act;
    uint16_t* pre;  // the sums, nullable
    long ldpre;
    // by expert: w is the first expert's
    const struct MxRowPlan* plan;
    const int* offsets;  // [experts + 1]
    int experts;
};
// Row tiles of a product by expert, made on the GPU from the experts' offsets: a tile starts at row `start` and writes rows first .. end - 1 of what it covers.
struct MxPlanTile {
    int expert, start, first, end;
};
struct MxRowPlan {
    uint32_t tiles, pad[3];
    MxPlanTile tile[1];
};
// Entries of a row plan, the same for all lanes.
typedef const __attribute__((address_space(4))) int const_int;
__device__ __forceinline__ uint32_t mx_plan_tiles(const MxRowPlan* p) { return __builtin_amdgcn_readfirstlane(*(const_int*)(uintptr_t)p); }
__device__ __forceinline__ MxPlanTile mx_plan_tile(const MxRowPlan* p, int i) {
    const const_int* t = (const_int*)(uintptr_t)(p->tile + i);
    return MxPlanTile{__builtin_amdgcn_readfirstlane(t[0]), __builtin_amdgcn_readfirstlane(t[1]), __builtin_amdgcn_readfirstlane(t[2]),
                      __builtin_amdgcn_readfirstlane(t[3])};
}
// Most tiles of at least 32 rows that a plan can have: whole ones, and for each expert with rows one that is not whole and one more where tiles start with whole
// groups of 32 rows and its first row is inside one.
inline long mx_plan_bound(long M, int experts, int tile_rows) { return M / tile_rows + 2 * (M < experts ? M : experts); }
inline size_t mx_plan_bytes(long M, int experts, int tile_rows) { return (sizeof(MxRowPlan) + mx_plan_bound(M, experts, tile_rows) * sizeof(MxPlanTile) + 255) / 256 * 256; }
int launch_mx_quantize(const void* x, int M, int K, long ldx, int dtype, void* mx, hipStream_t st);
int launch_mx_dequantize(const void* mx, int M, int K, int dtype, void* y, long ldy, hipStream_t st);
int launch_mx_pack(const uint8_t* codes, const uint8_t* scales, int M, int K, void* mx, hipStream_t st);
int launch_mx_unpack(const void* mx, int M, int K, uint8_t* codes, uint8_t* scales, hipStream_t st);
int launch_mx_experts_column_top(const void* mx, int experts, int N, int K, uint8_t* top, hipStream_t st);
int launch_mx_column_top(const void* mx, int rows, int K, uint8_t* top, hipStream_t st);
int launch_mx_gemm(const MxGemm& g, hipStream_t st);
int launch_mx_gemm_act(const MxGemm& g, bool gated, hipStream_t st);
int launch_mx_rows(const MxGemm& g, const void* x, long ldx, hipStream_t st);  // x: 16-bit activations, or null: g.a
int launch_mx_rows_act(const MxGemm& g, bool gated, hipStream_t st);
int launch_mx_few_rows(const MxGemm& g, bool gated, const void* x, long ldx, hipStream_t st);
bool mx_few_rows_takes(int M, int N, int K);
int launch_mx_experts(const MxGemm& g, bool gated, const void* x, long ldx, void* ws, hipStream_t st);
size_t mx_experts_workspace_bytes(long M, long N, long K, int experts);
bool mx_rows_takes(int M, int N);
bool mx_rows_quantizes(int M, int N, int K);
int launch_mx_experts_grad(const void* dy, int M, int N, long lddy, const void* w, const uint8_t* top, int K, int experts, const int* offsets, void* dx, long lddx,
                           int dtype, hipStream_t st);
int launch_mx_grad(const void* dy, int M, int N, long lddy, const void* w, const uint8_t* top, int K, void* dx, long lddx, int dtype, void* ws,
                   hipStream_t st);
size_t mx_grad_workspace_bytes(long M, long N, long K);
struct ActGrad {
    const uint16_t* dy;  // [M, O], O = N, gated N / 2
    long lddy;
    const uint16_t* pre;  // [M, N]
    long ldpre;
    int M, N, act;
    bool gated;
    uint16_t* da;
    long ldda;
    int dtype;
    float* dbias;    // nullable
    float* partial;  // workspace
};
int launch_act_grad(const ActGrad& a, hipStream_t st);
size_t act_grad_workspace_bytes(long M, long N, bool gated);

struct NormArgs {
    const uint16_t* x;
    long ldx;
    int M, C;
    const void* weight;  // nullable: 1
    const void* bias;    // nullable: 0
    int param_dtype;
    float eps;
    int dtype;
    float* mean;  // [M], nullable in the forward pass
    float* rstd;
    // forward
    uint16_t* y;
    long ldy;
    void* mx;
    // backward
    const uint16_t* dy;
    long lddy;
    const uint16_t* res;
    long ldr;
    uint16_t* dx;
    long lddx;
    float* dweight;  // nullable
    float* dbias;    // nullable
    float* partial;  // workspace
};
// Query and key heads: x [M, (q + k) D], rows of heads.
struct HeadArgs {
    const uint16_t* x;
    long ldx;
    int M, q, k, D;
    const void *qw, *kw;  // nullable: 1
    int param_dtype;
    float eps;
    bool norm;
    const uint4v* table;  // of every pair: fraction of a turn for one position (low word, high word), axis
    int pairs;            // 0: no rotation
    bool interleaved;
    const void* pos;  // [M, axes], 4 or 8 bytes each
    int pos_bytes, axes;
    long ldpos;
    int dtype;
    // forward
    uint16_t* y;
    long ldy;
    // backward
    const uint16_t* dy;
    long lddy;
    uint16_t* dx;
    long lddx;
    float *dq_weight, *dk_weight;  // nullable
    float* partial;                // workspace
    // set by the launcher: chunks of a row's heads, heads in each, waves' tasks in all
    FastDiv chunks;
    int per_chunk;
    uint32_t tasks;
};
int launch_heads(HeadArgs& a, bool grad, hipStream_t st);
size_t heads_grad_workspace_bytes(long M, int H, int D);

int launch_layer_norm(const NormArgs& a, hipStream_t st);
int launch_layer_norm_mx(const NormArgs& a, hipStream_t st);
size_t layer_norm_grad_workspace_bytes(long M, long C);
int launch_layer_norm_grad(const NormArgs& a, hipStream_t st);

}  // namespace mq

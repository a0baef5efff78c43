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
};
int launch_mx_quantize(const void* x, int M, int K, long ldx, int dtype, void* mx, hipStream_t st);
int launch_mx_dequantize(const void* mx, int M, int K, int dtype, void* y, long ldy, hipStream_t st);
int launch_mx_pack(const uint8_t* codes, const uint8_t* scales, int M, int K, void* mx, hipStream_t st);
int launch_mx_unpack(const void* mx, int M, int K, uint8_t* codes, uint8_t* scales, hipStream_t st);
int launch_mx_column_top(const void* mx, int rows, int K, uint8_t* top, hipStream_t st);
int launch_mx_gemm(const MxGemm& g, hipStream_t st);
int launch_mx_rows(const MxGemm& g, const void* x, long ldx, hipStream_t st);  // x: 16-bit activations, or null: g.a
bool mx_rows_takes(int M, int N);
bool mx_rows_quantizes(int M, int N, int K);
int launch_mx_grad(const void* dy, int M, int N, long lddy, const void* w, const uint8_t* top, int K, void* dx, long lddx, int dtype, void* ws,
                   hipStream_t st);
size_t mx_grad_workspace_bytes(long M, long N, long K);

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
int launch_layer_norm(const NormArgs& a, hipStream_t st);
int launch_layer_norm_mx(const NormArgs& a, hipStream_t st);
size_t layer_norm_grad_workspace_bytes(long M, long C);
int launch_layer_norm_grad(const NormArgs& a, hipStream_t st);

}  // namespace mq

// Conversion to and from microscaled 4-bit floats: quantise, dequantise, the interchange form, and the largest scale of every block column.
#include "mx_common.h"

namespace mq {

// A lane converts eight consecutive values; four lanes share a block, and a wave covers 8 rows x 64 columns at a time, so that it reads
// whole 128-byte pieces of eight rows and writes two of 128 bytes (8 neighbouring rows of one block column).  Four such steps, 256 columns, make the
// scale word of a row and block column.  Bound by memory: 2 bytes read and 17/32 written per value.
template <int DT>
__global__ __launch_bounds__(256) void mx_quantize_kernel(const uint16_t* x, int M, int K, long ldx, uint8_t* codes, uint8_t* scales,
                                                          int kc, int kq) {
    const int lane = threadIdx.x & 63, sub = threadIdx.x >> 6;
    const int g = blockIdx.y + blockIdx.z * 65535;  // group of 32 rows; a wave takes eight of them
    const int q = blockIdx.x;
    if ((long)g * 32 >= M) return;
    const int j = sub * 8 + (lane >> 3), kb = (lane >> 2) & 1, part = lane & 3;
    const long row = (long)g * 32 + j;
    const int k0 = q * 256 + (lane & 7) * 8;
    const uint16_t* p = x + row * ldx + k0;
    uint4v v[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const bool in = row < M && k0 + 64 * i < K;  // K % 32 == 0: a block is whole or absent
        v[i] = in ? load8_16(p + 64 * i, 8) : uint4v{0, 0, 0, 0};
    }
    uint32_t word = 0;
    uint8_t* tile = codes + ((long)g * kc + q * 4) * 1024 + (kb * 32 + j) * 16 + part * 4;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t s = mx_scale_byte(quad_max(mx_top_16<DT>(v[i])));
        uint32_t w = mx_codes_16<DT>(v[i], mx_scale_operand(s));
        if (s == 255u) w = 0;
        word |= s << (8 * i);
        if (q * 4 + i < kc) *(uint32_t*)(tile + (long)i * 1024) = w;
    }
    if (part == 0) *(uint32_t*)(scales + ((long)g * kq + q) * 256 + (kb * 32 + j) * 4) = word;
}

static dim3 rows_grid(int x, long groups) {
    const long z = (groups + 65534) / 65535;
    return dim3((unsigned)x, (unsigned)(z > 1 ? 65535 : groups), (unsigned)z);
}

int launch_mx_quantize(const void* x, int M, int K, long ldx, int dtype, void* mx, hipStream_t st) {
    const MxView v = mx_view(mx, M, K);
    const dim3 grid = rows_grid(v.kq, v.groups);
    uint8_t *codes = (uint8_t*)v.codes, *scales = (uint8_t*)v.scales;
    if (dtype == MQ_F16)
        mx_quantize_kernel<MQ_F16><<<grid, 256, 0, st>>>((const uint16_t*)x, M, K, ldx, codes, scales, v.kc, v.kq);
    else
        mx_quantize_kernel<MQ_BF16><<<grid, 256, 0, st>>>((const uint16_t*)x, M, K, ldx, codes, scales, v.kc, v.kq);
    MQ_HIP_CHECK_LAUNCH();
    return MQ_OK;
}

// The way back, in the same order of lanes: exact in both types except where the value leaves the range of fp16.
template <int DT>
__global__ __launch_bounds__(256) void mx_dequantize_kernel(const uint8_t* codes, const uint8_t* scales, int M, int K, int kc, int kq, uint16_t* y,
                                                            long ldy) {
    const int lane = threadIdx.x & 63, sub = threadIdx.x >> 6;
    const int g = blockIdx.y + blockIdx.z * 65535, q = blockIdx.x;
    if ((long)g * 32 >= M) return;
    const int j = sub * 8 + (lane >> 3), kb = (lane >> 2) & 1, part = lane & 3;
    const long row = (long)g * 32 + j;
    if (row >= M) return;
    const int k0 = q * 256 + (lane & 7) * 8;
    const uint32_t word = *(const uint32_t*)(scales + ((long)g * kq + q) * 256 + (kb * 32 + j) * 4);
    const uint8_t* tile = codes + ((long)g * kc + q * 4) * 1024 + (kb * 32 + j) * 16 + part * 4;
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = q * 4 + i < kc ? *(const uint32_t*)(tile + (long)i * 1024) : 0u;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if (k0 + 64 * i >= K) break;
        const float s = mx_scale_operand((word >> (8 * i)) & 255u);
        uint4v o;
        if constexpr (DT == MQ_F16) {
            o[0] = h2_bits(__builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w[i], s, 0));
            o[1] = h2_bits(__builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w[i], s, 1));
            o[2] = h2_bits(__builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w[i], s, 2));
            o[3] = h2_bits(__builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w[i], s, 3));
        } else {
            o[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w[i], s, 0));
            o[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w[i], s, 1));
            o[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w[i], s, 2));
            o[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w[i], s, 3));
        }
        uint16_t* to = y + row * ldy + k0 + 64 * i;
        if ((uintptr_t)to % 16 == 0)  // past the caches: 16384 x 640 0.7 of 11 us.  (Pieces of lines want them: such stores of unaligned rows take twice as long.)
            __builtin_nontemporal_store(o, (uint4v*)to);
        else
            store8_16(to, o, 8);
    }
}

int launch_mx_dequantize(const void* mx, int M, int K, int dtype, void* y, long ldy, hipStream_t st) {
    const MxView v = mx_view(mx, M, K);
    const dim3 grid = rows_grid(v.kq, v.groups);
    if (dtype == MQ_F16)
        mx_dequantize_kernel<MQ_F16><<<grid, 256, 0, st>>>(v.codes, v.scales, M, K, v.kc, v.kq, (uint16_t*)y, ldy);
    else
        mx_dequantize_kernel<MQ_BF16><<<grid, 256, 0, st>>>(v.codes, v.scales, M, K, v.kc, v.kq, (uint16_t*)y, ldy);
    MQ_HIP_CHECK_LAUNCH();
    return MQ_OK;
}

// Interchange form: codes [M, K/2] (code 2i in the low half of byte i), scales [M, K/32], both row after row.  A thread moves one block.
template <bool PACK>
__global__ __launch_bounds__(256) void mx_interchange_kernel(uint8_t* flat_codes, uint8_t* flat_scales, int M, int K, int kc, int kq, uint8_t* codes,
                                                             uint8_t* scales) {
    const int blocks = PACK ? kq * 8 : K / 32;  // the packer writes the padding too
    const long rows = PACK ? ((long)M + 31) / 32 * 32 : M;
    for (long t = (long)blockIdx.x * 256 + threadIdx.x; t < rows * blocks; t += (long)gridDim.x * 256) {
        const long row = t / blocks;
        const int b = (int)(t % blocks), c = b >> 1, kb = b & 1;
        const long g = row >> 5;
        const int L = kb * 32 + (int)(row & 31);
        const bool in = row < M && b < K / 32;
        uint8_t* sp = scales + (g * kq + (c >> 2)) * 256 + L * 4 + (c & 3);
        uint8_t* cp = codes + (g * kc + c) * 1024 + L * 16;
        uint8_t* fp = flat_codes + row * (K / 2) + b * 16;
        if constexpr (PACK) {
            *sp = in ? flat_scales[row * (K / 32) + b] : 0;
            if (c < kc) {
                const bool nan = in && *sp == 255;  // one form of a block that stands for NaN
                for (int i = 0; i < 16; ++i) cp[i] = in && !nan ? fp[i] : 0;
            }
        } else {
            flat_scales[row * (K / 32) + b] = *sp;
            for (int i = 0; i < 16; ++i) fp[i] = cp[i];
        }
    }
}

template <bool PACK>
static int interchange(uint8_t* fc, uint8_t* fs, int M, int K, const MxView& v, hipStream_t st) {
    const long n = ((long)M + 31) / 32 * 32 * v.kq * 8;
    const unsigned grid = (unsigned)((n + 255) / 256 < 65536 ? (n + 255) / 256 : 65536);
    mx_interchange_kernel<PACK><<<grid, 256, 0, st>>>(fc, fs, M, K, v.kc, v.kq, (uint8_t*)v.codes, (uint8_t*)v.scales);
    MQ_HIP_CHECK_LAUNCH();
    return MQ_OK;
}
int launch_mx_pack(const uint8_t* codes, const uint8_t* scales, int M, int K, void* mx, hipStream_t st) {
    return interchange<true>((uint8_t*)codes, (uint8_t*)scales, M, K, mx_view(mx, M, K), st);
}
int launch_mx_unpack(const void* mx, int M, int K, uint8_t* codes, uint8_t* scales, hipStream_t st) {
    return interchange<false>(codes, scales, M, K, mx_view(mx, M, K), st);
}

// top[b] = largest scale byte below 255 of block column b (0 if there is none).  A workgroup takes the eight block columns of a scale word column.
__global__ __launch_bounds__(256) void mx_column_top_kernel(const uint8_t* scales, int groups, int kq, int blocks, uint8_t* top) {
    const int q = blockIdx.x, lane = threadIdx.x & 63, sub = threadIdx.x >> 6;
    uint32_t best[4] = {0, 0, 0, 0};
    for (int g = sub; g < groups; g += 4) {
        const uint32_t w = *(const uint32_t*)(scales + ((long)g * kq + q) * 256 + lane * 4);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t s = (w >> (8 * i)) & 255u;
            if (s != 255u && s > best[i]) best[i] = s;
        }
    }
    __shared__ uint32_t part[4][64][4];
#pragma unroll
    for (int i = 0; i < 4; ++i) part[sub][lane][i] = best[i];
    __syncthreads();
    if (threadIdx.x < 8) {  // block column 2 i + kb
        const int i = threadIdx.x >> 1, kb = threadIdx.x & 1;
        uint32_t m = 0;
        for (int s = 0; s < 4; ++s)
            for (int j = 0; j < 32; ++j) m = part[s][kb * 32 + j][i] > m ? part[s][kb * 32 + j][i] : m;
        const int b = q * 8 + threadIdx.x;
        if (b < blocks) top[b] = (uint8_t)m;
    }
}
int launch_mx_column_top(const void* mx, int rows, int K, uint8_t* top, hipStream_t st) {
    const MxView v = mx_view(mx, rows, K);
    mx_column_top_kernel<<<v.kq, 256, 0, st>>>(v.scales, v.groups, v.kq, K / 32, top);
    MQ_HIP_CHECK_LAUNCH();
    return MQ_OK;
}

}  // namespace mq

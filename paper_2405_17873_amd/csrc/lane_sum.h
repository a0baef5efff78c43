// Sums over lanes.
#pragma once
#include "mq_common.h"

namespace mq {

template <int CTRL>
__device__ __forceinline__ float dpp(float v) {
    return __uint_as_float((uint32_t)__builtin_amdgcn_mov_dpp((int)__float_as_uint(v), CTRL, 0xF, 0xF, true));
}
__device__ __forceinline__ float swap_sum16(float v) {
    const auto p = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __uint_as_float((uint32_t)p[0]) + __uint_as_float((uint32_t)p[1]);
}
__device__ __forceinline__ float swap_sum32(float v) {
    const auto p = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __uint_as_float((uint32_t)p[0]) + __uint_as_float((uint32_t)p[1]);
}
// Sum over aligned runs of LANES lanes (a power of two up to 64), the same bits in each of them.
template <int LANES>
__device__ __forceinline__ float lane_sum(float v) {
    if constexpr (LANES >= 2) v += dpp<0xB1>(v);    // lanes 1,0,3,2 of four
    if constexpr (LANES >= 4) v += dpp<0x4E>(v);    // lanes 2,3,0,1
    if constexpr (LANES >= 8) v += dpp<0x141>(v);   // mirror of eight
    if constexpr (LANES >= 16) v += dpp<0x140>(v);  // mirror of sixteen
    if constexpr (LANES >= 32) v = swap_sum16(v);
    if constexpr (LANES >= 64) v = swap_sum32(v);
    return v;
}

}  // namespace mq

// The rows of experts, from their offsets on the GPU: tiles of rows, counted by a wave, 64 experts at a time.
#pragma once
#include "mx_common.h"

namespace mq {

struct ExpertWalk {
    int base = 0, before = 0, reach = 0;   // first expert of this turn; tiles, and furthest end, of the turns before
    int first, end, start, count, upto;    // of this lane's expert: rows, the first tile's first row, tiles, and tiles up to and with it in this turn
    int turn_tiles, turn_reach;

    static __device__ __forceinline__ int scan_max(int v) {
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const int o = __shfl_up(v, d);
            if ((int)(threadIdx.x & 63) >= d && o > v) v = o;
        }
        return v;
    }
    static __device__ __forceinline__ int scan_sum(int v) {
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const int o = __shfl_up(v, d);
            if ((int)(threadIdx.x & 63) >= d) v += o;
        }
        return v;
    }
    // `below`: 31 for tiles that start with whole groups of 32 rows, or 0.  Offsets that fall, or leave 0 .. M, are held at what came before, so that no row
    // has two experts.
    __device__ __forceinline__ void load(const int* offsets, int experts, int M, int tile_rows, int below) {
        const int lane = threadIdx.x & 63, e = base + lane;
        first = e < experts ? offsets[e] : 0, end = e < experts ? offsets[e + 1] : 0;
        first = first < 0 ? 0 : first > M ? M : first;
        end = end < 0 ? 0 : end > M ? M : end;
        int far = scan_max(end);
        far = far > reach ? far : reach;
        const int last = __shfl_up(far, 1), hold = lane ? last : reach;
        first = first > hold ? first : hold;
        start = first & ~below;
        count = e < experts && end > first ? (end - start + tile_rows - 1) / tile_rows : 0;
        upto = scan_sum(count);
        turn_tiles = __builtin_amdgcn_readlane(upto, 63);
        turn_reach = __builtin_amdgcn_readlane(far, 63);
    }
    __device__ __forceinline__ void next() {
        base += 64;
        before += turn_tiles;
        reach = turn_reach;
    }
    // The tile with this number, which is one of this turn's.
    __device__ __forceinline__ MxPlanTile tile(int number, int tile_rows) const {
        const int k = number - before;
        const int lane = __builtin_ctzll(__ballot(upto > k));
        const int i = k - (__builtin_amdgcn_readlane(upto, lane) - __builtin_amdgcn_readlane(count, lane));
        return MxPlanTile{base + lane, __builtin_amdgcn_readlane(start, lane) + i * tile_rows, __builtin_amdgcn_readlane(first, lane), __builtin_amdgcn_readlane(end, lane)};
    }
};

}  // namespace mq

// Row groups of a grouped product, found on the GPU from their cumulative ends.
//
// Group g holds the rows from where group g - 1 ends to ends[g]; a value below
// an earlier end counts as that end (an empty group) and one past T as T, so
// whatever the array holds, the groups are disjoint ranges of [0, T).  The rows
// past the last end are one more group, G, without a B.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace xtc {

struct RowTile {
    int group;        // G: rows past every group (zeros); -1: no such tile
    int row0, rows;   // rows row0 .. row0 + rows - 1 (at most the tile's height)
};

// Lane l's value of a running maximum or sum over the lanes up to l.
__device__ __forceinline__ int scan_max(int v, int lane) {
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
        const int u = __shfl_up(v, d, 64);
        if (lane >= d) v = v > u ? v : u;
    }
    return v;
}
__device__ __forceinline__ int scan_sum(int v, int lane) {
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
        const int u = __shfl_up(v, d, 64);
        if (lane >= d) v += u;
    }
    return v;
}

// Tile `index` of the groups' rows cut into tiles of BM, groups in order.
// Every lane of a wave calls it with the same index: 64 groups a step.  At
// most T / BM + G + 1 tiles exist.
template <int BM>
__device__ __forceinline__ RowTile find_row_tile(const int32_t *ends, int G, int T, int index) {
    const int lane = threadIdx.x & 63;
    int before = 0, prev = 0;       // tiles and rows of the groups of earlier steps
    for (int g0 = 0; g0 <= G; g0 += 64) {
        const int g = g0 + lane;
        int end = g < G ? ends[g] : T;
        end = end > T ? T : end;
        end = scan_max(end > prev ? end : prev, lane);
        int start = __shfl_up(end, 1, 64);
        if (lane == 0) start = prev;
        const int tiles = g <= G ? (end - start + BM - 1) / BM : 0;
        const int upto = scan_sum(tiles, lane);
        const bool mine = index >= before + upto - tiles && index < before + upto;
        const unsigned long long who = __ballot(mine);
        if (who) {
            const int l = __ffsll((long long)who) - 1;
            const int s = __shfl(start, l, 64), e = __shfl(end, l, 64), u = __shfl(upto - tiles, l, 64);
            const int row0 = s + (index - before - u) * BM;
            return RowTile{__builtin_amdgcn_readfirstlane(g0 + l), __builtin_amdgcn_readfirstlane(row0),
                           __builtin_amdgcn_readfirstlane(e - row0 < BM ? e - row0 : BM)};
        }
        before += __shfl(upto, 63, 64);
        prev = __shfl(end, 63, 64);
    }
    return RowTile{-1, 0, 0};
}

// The rows of group g (g < G).
__device__ __forceinline__ RowTile find_group(const int32_t *ends, int T, int g) {
    const int lane = threadIdx.x & 63;
    int start = 0, end = 0;
    for (int i0 = 0; i0 <= g; i0 += 64) {
        const int i = i0 + lane;
        int v = i <= g ? ends[i] : 0;
        v = v > T ? T : v < 0 ? 0 : v;
        const int upto = scan_max(v, lane);           // lanes past g repeat the last
        const int last = g - i0 < 63 ? g - i0 : 63;
        const int e = __shfl(upto, last, 64), s = last > 0 ? __shfl(upto, last - 1, 64) : 0;
        start = g - i0 <= 63 ? (end > s ? end : s) : 0;
        end = end > e ? end : e;
    }
    return RowTile{g, __builtin_amdgcn_readfirstlane(start), __builtin_amdgcn_readfirstlane(end - start)};
}

}  // namespace xtc

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

// The groups' rows cut into tiles of BM, groups in order: how many tiles there
// are (at most T / BM + G + 1) and which rows tile `index` holds.  Every lane of
// a wave calls it with the same arguments: 64 groups a step.
template <int BM>
struct RowTiles {
    const int32_t *ends;
    int G, T;
    int total;

    struct Step {
        int start, end, tiles, upto;    // of this lane's group; tiles of the step's groups up to it
    };
    // Groups g0 .. g0 + 63, the rows before them ending at prev.
    __device__ __forceinline__ Step step(int g0, int prev) const {
        const int lane = threadIdx.x & 63, g = g0 + lane;
        Step s;
        int end = g < G ? ends[g] : T;
        end = end > T ? T : end;
        s.end = scan_max(end > prev ? end : prev, lane);
        s.start = __shfl_up(s.end, 1, 64);
        if (lane == 0) s.start = prev;
        s.tiles = g <= G ? (s.end - s.start + BM - 1) / BM : 0;
        s.upto = scan_sum(s.tiles, lane);
        return s;
    }
    Step first;

    // (without ends: one group of all T rows)
    __device__ __forceinline__ RowTiles(const int32_t *ends_, int G_, int T_) : ends(ends_), G(G_), T(T_), first{} {
        if (!ends) {
            total = (T + BM - 1) / BM;
            return;
        }
        first = step(0, 0);
        total = __builtin_amdgcn_readlane(first.upto, 63);
        int prev = __builtin_amdgcn_readlane(first.end, 63);
        for (int g0 = 64; g0 <= G; g0 += 64) {
            const Step s = step(g0, prev);
            total += __builtin_amdgcn_readlane(s.upto, 63);
            prev = __builtin_amdgcn_readlane(s.end, 63);
        }
    }

    __device__ __forceinline__ RowTile find(int index) const {
        if (!ends) {
            const int row0 = index * BM;
            return RowTile{0, row0, T - row0 < BM ? T - row0 : BM};
        }
        Step s = first;
        int before = 0;
        for (int g0 = 0;; g0 += 64) {
            const unsigned long long who = __ballot(index >= before + s.upto - s.tiles && index < before + s.upto);
            if (who) {
                const int l = __ffsll((long long)who) - 1;
                const int first_tile = before + __builtin_amdgcn_readlane(s.upto - s.tiles, l);
                const int row0 = __builtin_amdgcn_readlane(s.start, l) + (index - first_tile) * BM;
                const int left = __builtin_amdgcn_readlane(s.end, l) - row0;
                return RowTile{g0 + l, row0, left < BM ? left : BM};
            }
            if (g0 + 64 > G) return RowTile{-1, 0, 0};
            before += __builtin_amdgcn_readlane(s.upto, 63);
            s = step(g0 + 64, __builtin_amdgcn_readlane(s.end, 63));
        }
    }
};

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
        const int e = __builtin_amdgcn_readlane(upto, last), s = last > 0 ? __builtin_amdgcn_readlane(upto, last - 1) : 0;
        start = g - i0 <= 63 ? (end > s ? end : s) : 0;
        end = end > e ? end : e;
    }
    return RowTile{g, start, end - start};
}

}  // namespace xtc

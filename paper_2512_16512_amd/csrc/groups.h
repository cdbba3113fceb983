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

// Of each 64 groups the one that is `index` % 64 th in length, the longest first
// (index < G; every lane of a wave calls it with the same arguments).
__device__ __forceinline__ RowTile find_by_length(const int32_t *ends, int G, int T, int index) {
    const int lane = threadIdx.x & 63;
    int prev = 0;
    for (int g0 = 0;; g0 += 64) {
        const int g = g0 + lane;
        const int v = g < G ? ends[g] : 0;
        int end = scan_max(v > T ? T : v, lane);
        end = end > prev ? end : prev;
        if (index - g0 >= 64) {
            prev = __builtin_amdgcn_readlane(end, 63);
            continue;
        }
        int start = __shfl_up(end, 1, 64);
        if (lane == 0) start = prev;
        const int rows = g < G ? end - start : -1;
        int longer = 0;
        const int n = G - g0 < 64 ? G - g0 : 64;
        for (int i0 = 0; i0 < n; i0 += 8) {
#pragma unroll
            for (int i = 0; i < 8; ++i) longer += __builtin_amdgcn_readlane(rows, i0 + i) > rows ? 1 : 0;
        }
        // equally long ones in their order
        const int at = index - g0, same = __builtin_amdgcn_readlane(scan_max(longer <= at ? longer : 0, lane), 63);
        const unsigned long long those = __ballot(longer == same);
        const int before = __builtin_amdgcn_mbcnt_hi((unsigned)(those >> 32), __builtin_amdgcn_mbcnt_lo((unsigned)those, 0));
        const int l = __ffsll((long long)__ballot(longer == same && before == at - same)) - 1;
        return RowTile{g0 + l, __builtin_amdgcn_readlane(start, l), __builtin_amdgcn_readlane(rows, l)};
    }
}

}  // namespace xtc

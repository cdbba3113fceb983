// What the kernels of the grouped and 8-bit products share: which tile of which
// member of the family a workgroup computes, and the store of its results.
//
// The matrix-core instructions take B's side (the columns of C) as their first
// operand and A's rows as their second, so that a lane's accumulators are four
// consecutive columns of one row of C, and an e4m3 row's scale is one value per
// lane: sum_k over a block of 128 is computed from zero, then added to the
// fp32 accumulators times the product of the two scales.
#pragma once

#include "groups.h"
#include "mfma_fp8.h"
#include "operators.h"
#include "tile_map.h"

namespace xtc {

// A tile of one member of the family.
struct Tile {
    const unsigned char *A, *B;   // row (or k) 0 of the tile's operands
    int64_t lda, ldb;             // bytes
    int m, n, k;                  // extents from the tile's corner (k: the whole reduction)
    const float *SA, *SB;
    unsigned char *C;
};

constexpr int kBand = 4;

enum Kind { kFp8, kBf16N, kBf16T, kWgrad };   // B [N, K] e4m3; bf16 [K, N]; bf16 [N, K]; both [T, .]

template <Kind KIND, int BM, int BN>
__device__ __forceinline__ bool find_tile(const GroupedArgs &p, Tile &t) {
    constexpr int E = KIND == kFp8 ? 1 : 2;
    const int tiles_n = (p.N + BN - 1) / BN;
    const int out = p.out_bf16 ? 2 : 4;
    const unsigned char *A = static_cast<const unsigned char *>(p.A), *B = static_cast<const unsigned char *>(p.B);
    unsigned char *C = static_cast<unsigned char *>(p.C);
    t.lda = p.lda * E;
    t.ldb = p.ldb * E;
    t.SA = t.SB = nullptr;
    if constexpr (KIND == kWgrad) {
        // rows of C: columns of A
        const int tiles_m = (p.K + BM - 1) / BM, per = tiles_m * tiles_n;
        const int g = (int)(blockIdx.x / per), r = (int)(blockIdx.x - (unsigned)g * per);
        const int m0 = r / tiles_n * BM, n0 = r % tiles_n * BN;
        const RowTile w = find_group(p.ends, (int)p.T, g);
        t.A = A + w.row0 * t.lda + (int64_t)m0 * E;
        t.B = B + w.row0 * t.ldb + (int64_t)n0 * E;
        t.m = p.K - m0;
        t.n = p.N - n0;
        t.k = w.rows;
        t.C = C + (g * p.stride_c + m0 * p.ldc + n0) * out;
        return true;
    }
    // Tiles that run together on one XCD are neighbours: bands of kBand row
    // tiles, walked column by column.
    RowTile w;
    int n0;
    if (p.ends) {
        const RowTiles<BM> tiles(p.ends, p.G, (int)p.T);
        if (blockIdx.x >= (unsigned)(tiles.total * tiles_n)) return false;   // (the launch holds the most there can be)
        int im, in;
        tile_coords((int)blockIdx.x, tiles.total * tiles_n, tiles.total, tiles_n, kBand, 1, im, in);
        n0 = in * BN;
        w = tiles.find(im);
    } else {
        int im, in;
        tile_coords((int)blockIdx.x, (int)gridDim.x, (int)((p.T + BM - 1) / BM), tiles_n, kBand, 1, im, in);
        n0 = in * BN;
        const int row0 = im * BM;
        w = RowTile{0, row0, p.T - row0 < BM ? (int)(p.T - row0) : BM};
    }
    const bool none = w.group >= p.G;
    t.A = A + w.row0 * t.lda;
    t.B = none ? B : B + w.group * p.stride_b * E + (KIND == kBf16N ? (int64_t)n0 * E : n0 * t.ldb);
    t.m = w.rows;
    t.n = p.N - n0;
    t.k = none ? 0 : p.K;
    if constexpr (KIND == kFp8) {
        t.SA = p.SA + w.row0 * p.ldsa;
        t.SB = none ? p.SB : p.SB + w.group * p.stride_sb + n0 / kScaleBlock * p.ldsb;
    }
    t.C = C + (w.row0 * p.ldc + n0) * out;
    return true;
}

// Writes v[0 .. 3], the columns n .. n + 3 of a row of C at `c`, of which `left` exist.
__device__ __forceinline__ void write4(const GroupedArgs &p, unsigned char *c, int n, int left, float (&v)[4]) {
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (p.relu && v[i] < 0.f) v[i] = 0.f;
    if (p.out_bf16) {
        __bf16 t[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) t[i] = (__bf16)v[i];
        __bf16 *d = reinterpret_cast<__bf16 *>(c) + n;
        if (left >= 4) {
            __builtin_memcpy(d, t, 8);
        } else {
#pragma unroll
            for (int i = 0; i < 3; ++i)
                if (i < left) d[i] = t[i];
        }
    } else {
        float *d = reinterpret_cast<float *>(c) + n;
        if (left >= 4) {
            __builtin_memcpy(d, v, 16);
        } else {
#pragma unroll
            for (int i = 0; i < 3; ++i)
                if (i < left) d[i] = v[i];
        }
    }
}

inline int64_t cdiv(int64_t a, int64_t b) { return (a + b - 1) / b; }

// Tiles of bm rows that a launch has to hold for whatever groups the GPU finds.
inline int64_t row_tiles(const GroupedArgs &a, int bm) { return a.ends ? a.T / bm + a.G + 1 : cdiv(a.T, bm); }

// Workgroups of BM x BN tiles.
template <Kind KIND>
int64_t tile_count(const GroupedArgs &a, int bm, int bn) {
    return (KIND == kWgrad ? cdiv(a.K, bm) * a.G : row_tiles(a, bm)) * cdiv(a.N, bn);
}

// The kernels of one file each.  launch_any takes every call; launch_tile those
// that tile_takes.
template <Kind KIND>
xtc_status launch_any(const GroupedArgs &a, hipStream_t s);
template <Kind KIND>
bool tile_takes(const GroupedArgs &a);
template <Kind KIND>
xtc_status launch_tile(const GroupedArgs &a, hipStream_t s);

}  // namespace xtc

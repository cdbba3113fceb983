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

// Where a tile lies: what its operands' addresses follow from.
struct Place {
    int group;          // p.G: rows past every group, without a B
    int row0, rows;     // of the group's rows: the tile's, or for a weights' gradient all of them
    int m0, n0;         // corner in C (m0: weights' gradient only)
};

template <Kind KIND>
__device__ __forceinline__ Tile make_tile(const GroupedArgs &p, const Place &w) {
    constexpr int E = KIND == kFp8 ? 1 : 2;
    const int out = p.out_bf16 ? 2 : 4;
    const bool none = w.group >= p.G;
    const unsigned char *A = static_cast<const unsigned char *>(p.A), *B = static_cast<const unsigned char *>(p.B);
    Tile t;
    t.lda = p.lda * E;
    t.ldb = p.ldb * E;
    t.SA = t.SB = nullptr;
    t.n = p.N - w.n0;
    t.A = A + w.row0 * t.lda;
    unsigned char *C = static_cast<unsigned char *>(p.C);
    if constexpr (KIND == kWgrad) {
        t.A += (int64_t)w.m0 * E;
        t.B = B + w.row0 * t.ldb + (int64_t)w.n0 * E;
        t.m = p.K - w.m0;
        t.k = w.rows;
        t.C = C + (w.group * p.stride_c + w.m0 * p.ldc + w.n0) * out;
    } else {
        t.B = none ? B : B + w.group * p.stride_b * E + (KIND == kBf16N ? (int64_t)w.n0 * E : w.n0 * t.ldb);
        t.m = w.rows;
        t.k = none ? 0 : p.K;
        if constexpr (KIND == kFp8) {
            t.SA = p.SA + w.row0 * p.ldsa;
            t.SB = none ? p.SB : p.SB + w.group * p.stride_sb + w.n0 / kScaleBlock * p.ldsb;
        }
        t.C = C + (w.row0 * p.ldc + w.n0) * out;
    }
    return t;
}

// The tiles of a product, BM x BN each, in an order in which neighbours share
// operands: bands of kBand row tiles, walked column by column.
template <Kind KIND, int BM, int BN>
struct TileOrder {
    const GroupedArgs &p;
    RowTiles<BM> rows;        // (of a product with groups)
    int tiles_n, per, total;

    __device__ __forceinline__ TileOrder(const GroupedArgs &p_)
        : p(p_), rows(KIND == kWgrad ? nullptr : p_.ends, p_.G, (int)p_.T) {
        tiles_n = (p.N + BN - 1) / BN;
        per = KIND == kWgrad ? (p.K + BM - 1) / BM * tiles_n : 0;
        total = KIND == kWgrad ? p.G * per : rows.total * tiles_n;
    }
    __device__ __forceinline__ Place at(int id) const {
        if constexpr (KIND == kWgrad) {
            const int g = id / per, r = id - g * per;
            const RowTile w = find_by_length(p.ends, p.G, (int)p.T, g);
            return Place{w.group, w.row0, w.rows, r / tiles_n * BM, r % tiles_n * BN};
        } else {
            int im, in;
            tile_coords(id, total, rows.total, tiles_n, kBand, 0, im, in);
            const RowTile w = rows.find(im);
            return Place{w.group, w.row0, w.rows, 0, in * BN};
        }
    }
};

// The id of this workgroup's tile, or -1 (a launch holds the most tiles there
// can be).  Workgroups go to the 8 XCDs in turn; each XCD gets an equal run of
// neighbouring tiles, but of a weights' gradient, whose tiles are not equally
// long, every eighth, the longest groups' first (16384 rows over 16 uneven groups,
// 1024 x 2048 each, tiles of 128x256: in the groups' order a tenth longer).
template <Kind KIND>
__device__ __forceinline__ int tile_id(int total) {
    const int b = (int)blockIdx.x, x = b & 7, j = b >> 3, q = total >> 3, rem = total & 7;
    if (KIND == kWgrad) return b < total ? b : -1;
    return j < q + (x < rem ? 1 : 0) ? x * q + (x < rem ? x : rem) + j : -1;
}

__device__ __forceinline__ float relu_if(int relu, float v) { return relu && v < 0.f ? 0.f : v; }

// Writes v[0 .. 3], the columns n .. n + 3 of a row of C at `c`, of which `left` exist.
__device__ __forceinline__ void write4(const GroupedArgs &p, unsigned char *c, int n, int left, float (&v)[4]) {
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

// 16 bytes of results to p, of which the first `left` exist.
template <typename T, int N>
__device__ __forceinline__ void store_past_caches(T *p, const T (&v)[N], int left) {
    static_assert(N * sizeof(T) == 16, "16 bytes");
    typedef unsigned u32x4s __attribute__((ext_vector_type(4), aligned(2)));
    if (left >= N) {
        u32x4s q;
        __builtin_memcpy(&q, v, 16);
        __builtin_nontemporal_store(q, reinterpret_cast<u32x4s *>(p));
    } else {
#pragma unroll
        for (int i = 0; i < N - 1; ++i)
            if (i < left) p[i] = v[i];
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

// A compiled kernel and what a launch of it takes, in microseconds: with n tiles
// on 256 CUs of per_cu workgroups each, every round costs `fixed` (the first
// data's way and the results') and for each stage of k (128 bytes) `one` where
// a CU holds one workgroup (`cold` with weights that come from memory), `full`
// where it holds per_cu.
struct Choice {
    int bm, bn, per_cu;
    float one, cold, full, fixed;
    bool dense_only;        // for products without groups
    xtc_status (*launch)(const GroupedArgs &, hipStream_t);
};

// The kernels of one file each, fp32 sums of e4m3 products where `wide`.
// launch_any takes every call, the others those that aligned_rows() takes.
template <Kind KIND>
xtc_status launch_any(const GroupedArgs &a, hipStream_t s);
template <Kind KIND>
const Choice *tile_choices(bool wide, int *count);
template <Kind KIND>
const Choice *stream_choices(bool wide, int *count);

}  // namespace xtc

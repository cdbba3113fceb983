// Products with the rows of A in groups, each with its own B, and the 8-bit
// products with block scales (of one group or several).
//
// The matrix-core instructions take B's side (the columns of C) as their first
// operand and A's rows as their second, so that a lane's accumulators are four
// consecutive columns of one row of C, and an e4m3 row's scale is one value per
// lane: sum_k over a block of 128 is computed from zero, then added to the
// fp32 accumulators times the product of the two scales.
#include "groups.h"
#include "mfma_fp8.h"
#include "operators.h"

namespace xtc {
namespace {

// A tile of one member of the family.
struct Tile {
    const unsigned char *A, *B;   // row (or k) 0 of the tile's operands
    int64_t lda, ldb;             // bytes
    int m, n, k;                  // extents from the tile's corner (k: the whole reduction)
    const float *SA, *SB;
    unsigned char *C;
};

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
    const int im = (int)(blockIdx.x / tiles_n), n0 = (int)(blockIdx.x - (unsigned)im * tiles_n) * BN;
    RowTile w;
    if (p.ends) {
        w = find_row_tile<BM>(p.ends, p.G, (int)p.T, im);
    } else {
        const int row0 = im * BM;
        w = RowTile{0, row0, p.T - row0 < BM ? (int)(p.T - row0) : BM};
    }
    if (w.group < 0) return false;
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

// Writes v[0 .. 3], the columns n .. n + 3 of a row of C at `c`.
__device__ __forceinline__ void write4(const GroupedArgs &p, unsigned char *c, int n, int left, float (&v)[4]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if (p.relu && v[i] < 0.f) v[i] = 0.f;
        if (i < left) {
            if (p.out_bf16) reinterpret_cast<__bf16 *>(c)[n + i] = (__bf16)v[i];
            else reinterpret_cast<float *>(c)[n + i] = v[i];
        }
    }
}

// Rows, columns and strides of any alignment: operands through registers into
// one padded LDS buffer, k innermost.  64 x 64 tiles of four 32 x 32 waves.
template <Kind KIND>
__global__ void __launch_bounds__(256) grouped_any_kernel(GroupedArgs p) {
    constexpr bool FP8 = KIND == kFp8;
    constexpr int BM = 64, BN = 64, ROW = 128 + 16, E = FP8 ? 1 : 2, BK = 128 / E;
    __shared__ __attribute__((aligned(16))) unsigned char As[BM * ROW], Bs[BN * ROW];
    Tile t;
    if (!find_tile<KIND, BM, BN>(p, t)) return;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int wm = (wave >> 1) * 32, wn = (wave & 1) * 32, l16 = lane & 15, g4 = lane >> 4;

    // One operand's tile: 64 rows of 128 bytes of k.
    auto stage = [&](unsigned char *s, const unsigned char *src, int64_t ld, int rows, int k0, bool k_rows) {
        if (!k_rows) {
#pragma unroll
            for (int q = 0; q < 2; ++q) {
                const int row = (tid >> 3) + q * 32, c = (tid & 7) * 16;
                const int valid = row < rows ? (t.k - k0) * E - c : 0;
                unsigned char v[16];
                const unsigned char *g = src + row * ld + (int64_t)k0 * E + c;
                if (valid >= 16) {
                    __builtin_memcpy(v, g, 16);
                } else {
#pragma unroll
                    for (int i = 0; i < 16; ++i) v[i] = i < valid ? g[i] : 0;
                }
                __builtin_memcpy(__builtin_assume_aligned(s + row * ROW + c, 16), v, 16);
            }
        } else {
            // bf16 with one k a row: eight columns at a time, turned
#pragma unroll
            for (int q = 0; q < 2; ++q) {
                const int k = (tid >> 3) + q * 32, c = (tid & 7) * 8;
                const int valid = k0 + k < t.k ? rows - c : 0;
                unsigned short v[8];
                const unsigned char *g = src + (int64_t)(k0 + k) * ld + c * 2;
                if (valid >= 8) {
                    __builtin_memcpy(v, g, 16);
                } else {
#pragma unroll
                    for (int i = 0; i < 8; ++i)
                        v[i] = i < valid ? reinterpret_cast<const unsigned short *>(g)[i] : (unsigned short)0;
                }
#pragma unroll
                for (int i = 0; i < 8; ++i) *reinterpret_cast<unsigned short *>(s + (c + i) * ROW + k * 2) = v[i];
            }
        }
    };

    f32x4 acc[2][2] = {};
    for (int k0 = 0; k0 < t.k; k0 += BK) {
        stage(As, t.A, t.lda, t.m, k0, KIND == kWgrad);
        stage(Bs, t.B, t.ldb, t.n, k0, KIND == kBf16N || KIND == kWgrad);
        __syncthreads();
        if constexpr (FP8) {
            // (widened: fp32 sums whatever C's type)
            u16x8 a[2][4], b[2][4];
            float sa[2];
            const int kb = k0 / kScaleBlock;
            const float sb = t.SB[kb];
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const int row = wm + i * 16 + l16;
                const i32x8 qa = read_32_bytes(As + row * ROW + g4 * 32, 16);
                const i32x8 qb = read_32_bytes(Bs + (wn + i * 16 + l16) * ROW + g4 * 32, 16);
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    a[i][q] = widen_fp8((unsigned)qa[2 * q], (unsigned)qa[2 * q + 1]);
                    b[i][q] = widen_fp8((unsigned)qb[2 * q], (unsigned)qb[2 * q + 1]);
                }
                sa[i] = row < t.m ? t.SA[row * p.ldsa + kb] * sb : 0.f;
            }
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    f32x4 d = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                    for (int q = 0; q < 4; ++q) d = Bf16Mfma<16>::mma(b[j][q], a[i][q], d);
#pragma unroll
                    for (int r = 0; r < 4; ++r) acc[i][j][r] += d[r] * sa[i];
                }
        } else {
#pragma unroll
            for (int kk = 0; kk < 2; ++kk) {
                u16x8 a[2], b[2];
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    a[i] = *reinterpret_cast<const u16x8 *>(As + (wm + i * 16 + l16) * ROW + kk * 64 + g4 * 16);
                    b[i] = *reinterpret_cast<const u16x8 *>(Bs + (wn + i * 16 + l16) * ROW + kk * 64 + g4 * 16);
                }
#pragma unroll
                for (int i = 0; i < 2; ++i)
#pragma unroll
                    for (int j = 0; j < 2; ++j) acc[i][j] = Bf16Mfma<16>::mma(b[j], a[i], acc[i][j]);
            }
        }
        __syncthreads();
    }
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const int m = wm + i * 16 + l16, n = wn + j * 16 + 4 * g4;
            if (m >= t.m) continue;
            float v[4];
#pragma unroll
            for (int r = 0; r < 4; ++r) v[r] = acc[i][j][r];
            write4(p, t.C + m * p.ldc * (p.out_bf16 ? 2 : 4), n, t.n - n, v);
        }
}

int64_t cdiv(int64_t a, int64_t b) { return (a + b - 1) / b; }

// Tiles of bm rows that a launch has to hold for whatever groups the GPU finds.
int64_t row_tiles(const GroupedArgs &a, int bm) { return a.ends ? a.T / bm + a.G + 1 : cdiv(a.T, bm); }

template <Kind KIND>
xtc_status launch_any(const GroupedArgs &a, hipStream_t s) {
    const int64_t tiles = KIND == kWgrad ? cdiv(a.K, 64) * a.G : row_tiles(a, 64);
    if (tiles * cdiv(a.N, 64) >= kMostGroups) return XTC_ERR_TOO_LARGE;
    grouped_any_kernel<KIND><<<(unsigned)(tiles * cdiv(a.N, 64)), 256, 0, s>>>(a);
    return hip_status(hipGetLastError());
}

}  // namespace

xtc_status launch_grouped_fp8(const GroupedArgs &a, hipStream_t s) { return launch_any<kFp8>(a, s); }
xtc_status launch_grouped_bf16(const GroupedArgs &a, bool b_rows_n, hipStream_t s) {
    return b_rows_n ? launch_any<kBf16T>(a, s) : launch_any<kBf16N>(a, s);
}
xtc_status launch_grouped_wgrad(const GroupedArgs &a, hipStream_t s) { return launch_any<kWgrad>(a, s); }

}  // namespace xtc

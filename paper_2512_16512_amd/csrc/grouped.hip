// Products with the rows of A in groups, each with its own B, and the 8-bit
// products with block scales (of one group or several): the choice of the
// kernel, and the kernel for operands of any alignment.
#include "grouped.h"

namespace xtc {
namespace {

// Rows, columns and strides of any alignment: operands through registers into
// one padded LDS buffer, k innermost.  64 x 64 tiles of four 32 x 32 waves.
template <Kind KIND>
__global__ void __launch_bounds__(256) grouped_any_kernel(GroupedArgs p) {
    constexpr bool FP8 = KIND == kFp8;
    constexpr int BM = 64, BN = 64, ROW = 128 + 16, E = FP8 ? 1 : 2, BK = 128 / E;
    __shared__ __attribute__((aligned(16))) unsigned char As[BM * ROW], Bs[BN * ROW];
    const TileOrder<KIND, BM, BN> order(p);
    const int id = tile_id<KIND>(order.total);
    if (id < 0) return;
    const Tile t = make_tile<KIND>(p, order.at(id));
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
            for (int r = 0; r < 4; ++r) v[r] = relu_if(p.relu, acc[i][j][r]);
            write4(p, t.C + m * p.ldc * (p.out_bf16 ? 2 : 4), n, t.n - n, v);
        }
}

}  // namespace

template <Kind KIND>
xtc_status launch_any(const GroupedArgs &a, hipStream_t s) {
    const int64_t tiles = tile_count<KIND>(a, 64, 64);
    if (tiles >= kMostGroups) return XTC_ERR_TOO_LARGE;
    grouped_any_kernel<KIND><<<(unsigned)tiles, 256, 0, s>>>(a);
    return hip_status(hipGetLastError());
}

namespace {

bool aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }

// 16-byte aligned rows, whole 16-byte chunks of k where they run along it, and
// strides that keep the offsets within a tile in 31 bits.
template <Kind KIND>
bool aligned_rows(const GroupedArgs &a) {
    const int64_t e = KIND == kFp8 ? 1 : 2, most = (int64_t(1) << 31) / 257;
    if (!aligned16(a.A) || !aligned16(a.B) || a.lda * e % 16 || a.ldb * e % 16 || a.stride_b * e % 16) return false;
    if (KIND != kWgrad && a.K * e % 16) return false;
    return a.lda * e < most && a.ldb * e < most && a.ldsa * 4 < most && a.ldsb * 4 < most;
}

// The estimate of a launch.  How a group's rows fall into tiles only the GPU
// knows: half a tile a group is taken to be empty.
template <Kind KIND>
double estimate_us(const Choice &c, const GroupedArgs &a) {
    double rows, k;
    if (KIND == kWgrad) {
        rows = (double)cdiv(a.K, c.bm) * a.G;
        k = (double)a.T / a.G;
    } else {
        const double each = (double)a.T / a.G / c.bm + .5;
        rows = a.ends ? a.G * (each > 1 ? each : 1) : (double)cdiv(a.T, c.bm);
        k = a.K;
    }
    const double stages = k * (KIND == kFp8 ? 1 : 2) / 128, slots = 256. * c.per_cu;
    const int64_t n = (int64_t)(rows * cdiv(a.N, c.bn)), whole = (int64_t)(n / slots);
    const int64_t rest = n - (int64_t)(whole * slots), held = cdiv(rest, 256);
    double us = whole * (stages * c.full + c.fixed);
    if (held > 0) {
        const double last = stages * (held > 1 ? c.one + (c.full - c.one) * (held - 1) / (c.per_cu - 1) : c.one) + c.fixed;
        // (where CUs hold several workgroups, those of a last, partial round begin as others end)
        us += whole > 0 && c.per_cu > 1 ? last / 2 : last;
    }
    return us;
}

template <Kind KIND>
xtc_status launch(const GroupedArgs &a, hipStream_t s) {
    if (!aligned_rows<KIND>(a)) return launch_any<KIND>(a, s);
    const bool wide = KIND == kFp8 && !a.out_bf16;
    const Choice *best = nullptr;
    double least = 0;
    auto look = [&](const Choice *c, int count) {
        for (int i = 0; i < count; ++i) {
            if (c[i].dense_only && a.ends) continue;
            const double us = estimate_us<KIND>(c[i], a);
            if (!best || us < least) {
                best = &c[i];
                least = us;
            }
        }
    };
    int count = 0;
    const Choice *tiles = tile_choices<KIND>(wide, &count);
    look(tiles, count);
    if constexpr (KIND != kWgrad) {
        const Choice *streams = stream_choices<KIND>(wide, &count);
        look(streams, count);
    }
    return best->launch(a, s);
}

}  // namespace

xtc_status launch_grouped_fp8(const GroupedArgs &a, hipStream_t s) { return launch<kFp8>(a, s); }
xtc_status launch_grouped_bf16(const GroupedArgs &a, bool b_rows_n, hipStream_t s) {
    return b_rows_n ? launch<kBf16T>(a, s) : launch<kBf16N>(a, s);
}
xtc_status launch_grouped_wgrad(const GroupedArgs &a, hipStream_t s) { return launch<kWgrad>(a, s); }

}  // namespace xtc

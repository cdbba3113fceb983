// Products with the rows of A in groups, each with its own B, and the 8-bit
// products with block scales (of one group or several): the choice of the
// kernel.
#include "grouped.h"

namespace xtc {
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
    if (KIND == kWgrad) {
        // Tiles of different lengths fill the ends of each other's rounds; those of the
        // longest group, taken to hold up to 4.5 times its share, last that long in any
        // case (16384 rows over 16 uneven groups, 1024 x 2048 each: tiles of 256x256 101 to
        // 120 us, 128x256 95 to 96; over equal ones 90 and 95).  With few groups the guess can
        // be wrong: 11424 rows over 4, 1472 x 1088, 85 us where 128x256 takes 70, the most
        // of 26 problems.
        const double rounds = n / slots, second = n > 256 && c.per_cu > 1 ? (n - 256) / (slots - 256) : 0;
        const double us = rounds >= 1 ? rounds * (stages * c.full + c.fixed) : stages * (c.one + (c.full - c.one) * second) + c.fixed;
        const double longest = stages * c.one * (a.G < 8 ? (1 + a.G) / 2. : 4.5) + c.fixed;
        return us > longest ? us : longest;
    }
    const int64_t rest = n - (int64_t)(whole * slots), held = cdiv(rest, 256);
    // Weights above 64 MB are taken to come from memory in every call (100 rows over
    // 32 groups, bf16, 2048 to 1024: tiles of 64x128 34 us, 32x64 27; their stages at
    // the rate of cached weights would have been 21 and 23).
    const bool from_memory = (double)a.G * a.N * a.K * (KIND == kFp8 ? 1 : 2) > 64e6;
    const double one = from_memory ? c.cold : c.one, full = c.per_cu > 1 ? c.full : one;
    double us = whole * (stages * full + c.fixed);
    if (held > 0) {
        const double last = stages * (held > 1 ? one + (full - one) * (held - 1) / (c.per_cu - 1) : one) + c.fixed;
        // (where CUs hold several workgroups, those of a last, partial round begin as others end)
        us += whole > 0 && c.per_cu > 1 ? last / 2 : last;
    }
    return us;
}

// The kernel of the least estimate among those for aligned rows, and its place:
// tiles first, then streams.
template <Kind KIND>
const Choice *choose(const GroupedArgs &a, int *place) {
    const bool wide = KIND == kFp8 && !a.out_bf16;
    const Choice *best = nullptr;
    double least = 0;
    int seen = 0;
    auto look = [&](const Choice *c, int count) {
        for (int i = 0; i < count; ++i, ++seen) {
            if (c[i].dense_only && a.ends) continue;
            const double us = estimate_us<KIND>(c[i], a);
            if (!best || us < least) {
                best = &c[i];
                *place = seen;
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
    return best;
}

template <Kind KIND>
xtc_status launch(const GroupedArgs &a, hipStream_t s) {
    int place;
    if (!aligned_rows<KIND>(a)) return launch_any<KIND>(a, s);
    return choose<KIND>(a, &place)->launch(a, s);
}

template <Kind KIND>
int kernel_place(const GroupedArgs &a, int *kernels) {
    const bool wide = KIND == kFp8 && !a.out_bf16;
    int count = 0, place = -1;
    tile_choices<KIND>(wide, &count);
    *kernels = count;
    if constexpr (KIND != kWgrad) {
        stream_choices<KIND>(wide, &count);
        *kernels += count;
    }
    if (aligned_rows<KIND>(a)) choose<KIND>(a, &place);
    return place;
}

}  // namespace

xtc_status launch_grouped_fp8(const GroupedArgs &a, hipStream_t s) { return launch<kFp8>(a, s); }
xtc_status launch_grouped_bf16(const GroupedArgs &a, bool b_rows_n, hipStream_t s) {
    return b_rows_n ? launch<kBf16T>(a, s) : launch<kBf16N>(a, s);
}
xtc_status launch_grouped_wgrad(const GroupedArgs &a, hipStream_t s) { return launch<kWgrad>(a, s); }

int grouped_kernel(const GroupedArgs &a, int kind, int *kernels) {
    switch (kind) {
        case kFp8: return kernel_place<kFp8>(a, kernels);
        case kBf16N: return kernel_place<kBf16N>(a, kernels);
        case kBf16T: return kernel_place<kBf16T>(a, kernels);
        default: return kernel_place<kWgrad>(a, kernels);
    }
}

}  // namespace xtc

// The linear layer: the choice of its kernel and splits, the join of the splits' sums, and the
// gradients of its activation and bias.
#include "linear.h"

namespace xtc {
namespace {

bool aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }

// 16-byte aligned rows, with a stride that keeps the offsets within a tile in 31 bits.
bool aligned_rows(const void *p, int64_t ld) { return aligned16(p) && ld % 8 == 0 && ld * 2 < (int64_t(1) << 31) / 257; }

// A kernel, the parts of the reduction it is launched with, and the operands that are first copied
// to rows that it can take.
struct Plan {
    const LinearChoice *choice;
    int splits, k_each, place;
    bool copy_a, copy_b;
    int64_t ld_a, ld_b;                          // of the copies
    int64_t part_bytes, a_bytes, b_bytes;        // of the workspace, one after the other
};

constexpr int kSplitStep = 128;      // parts of the reduction are whole stages of every kernel
constexpr int kMostSplits = 16;
constexpr double kJoinUs = 2.4, kJoinPartUs = .15;
// Bytes of the copies, whatever they would save: a workspace must not grow with the operands (1000000 x 4095 to 4096 asked
// for 8.2 GB).  Beyond it rows off 16 bytes run as they are, at half the rate (70000 x 4097 to 4096 4.3 ms, copied 2.2).
constexpr int64_t kMostCopied = int64_t(512) << 20;

int64_t padded(int64_t n) { return cdiv(n, 8) * 8; }
int64_t room(int64_t bytes) { return cdiv(bytes, 256) * 256; }

// Microseconds of a launch of n tiles with `stages` of k each: rounds of tiles, no less than the operands'
// way from memory, and the way of the splits' sums to memory and back.  (A call makes up its plan twice; 0.2 us each.)
double estimate_us(const LinearChoice &c, int64_t n, double stages, double memory, int splits, double sums) {
    const int64_t slots = 256 * c.per_cu, whole = n < slots ? 0 : n / slots, rest = n - whole * slots;
    double us = whole * (stages * (c.per_cu > 1 ? c.full : c.one) + c.fixed);
    if (rest > 0) {
        const int64_t held = (rest + 255) >> 8;
        const double stage = held > 1 ? c.one + (c.full - c.one) * (held - 1) / (c.per_cu - 1) : c.one * (c.fill + (1 - c.fill) * rest / 256);
        const double last = stages * stage + c.fixed;
        // (where CUs hold several workgroups, those of a last, partial round begin as others end)
        us += whole > 0 && c.per_cu > 1 ? .75 * last : last;
    }
    us = us > memory ? us : memory;
    if (splits > 1) us += kJoinUs + kJoinPartUs * splits + 8. * splits * sums / 12e6;
    return us;
}
double copy_us(double bytes) { return 3.5 + bytes / 3.2e6; }

template <Kind KIND>
Plan plan(const LinearArgs &a) {
    const int64_t rows = KIND == kWgrad ? a.K : a.T, reduce = KIND == kWgrad ? a.T : a.K;
    const int64_t some = reduce > 1 ? reduce : 1;
    // (rows along k are read in whole 16 bytes, what lies behind their end among it)
    const bool whole_k = KIND == kWgrad || a.K % 8 == 0;
    const bool a_fits = aligned_rows(a.A, a.lda) && whole_k, b_fits = aligned_rows(a.B, a.ldb) && (KIND == kBf16N || whole_k);
    Plan best = {};
    best.splits = 1;
    best.k_each = (int)(cdiv(some, kSplitStep) * kSplitStep);
    double least = 0;
    int seen = 0;
    const double size_a = (double)a.T * a.K, size_b = (KIND == kWgrad ? (double)a.T : (double)a.K) * a.N, sums = (double)rows * a.N;
    const double memory = 2 + (size_a + size_b) * 2 / 5e6;
    const double copying = a_fits && b_fits ? 0 : copy_us((a_fits ? 0 : 2 * size_a) + (b_fits ? 0 : 2 * size_b));
    const int64_t ld_a = padded(a.K), ld_b = KIND == kBf16T ? padded(a.K) : padded(a.N);
    const int64_t a_bytes = a_fits ? 0 : room(a.T * ld_a * 2);
    const int64_t b_bytes = b_fits ? 0 : room((KIND == kBf16T ? a.N : KIND == kWgrad ? a.T : a.K) * ld_b * 2);
    auto look = [&](const LinearChoice *c, int count, bool copies) {
        for (int i = 0; i < count; ++i, ++seen) {
            const uint32_t bm = (uint32_t)c[i].bm, bn = (uint32_t)c[i].bn;
            const int64_t tiles = (int64_t)(((uint32_t)rows + bm - 1) / bm) * (((uint32_t)a.N + bn - 1) / bn);
            for (int want = 1, last = 0; want <= kMostSplits; want *= 2) {
                const uint32_t each = ((uint32_t)some + want * kSplitStep - 1) / (want * kSplitStep) * kSplitStep;
                const int splits = (int)(((uint32_t)some + each - 1) / each);
                // (nothing is gained by splits of tiles that fill the CUs)
                if (want > 1 && (splits < 2 || each < 256 || tiles * last >= 256 * c[i].per_cu)) break;
                last = splits;
                double us = estimate_us(c[i], tiles * splits, (double)(((each < some ? each : (uint32_t)some) + 63) / 64), memory, splits, sums);
                if (copies) us += copying;
                if (best.choice && us >= least) continue;
                Plan w = {};
                w.choice = &c[i];
                w.splits = splits;
                w.k_each = (int)each;
                w.place = seen;
                w.ld_a = ld_a;
                w.ld_b = ld_b;
                if (copies) w.a_bytes = a_bytes;
                if (copies) w.b_bytes = b_bytes;
                w.copy_a = w.a_bytes > 0;
                w.copy_b = w.b_bytes > 0;
                if (splits > 1) w.part_bytes = room(4 * (int64_t)splits * rows * a.N);
                best = w;
                least = us;
            }
        }
    };
    int count = 0;
    if (!a_fits || !b_fits) {
        const LinearChoice *any = linear_any_choices<KIND>(&count);
        look(any, count, false);
    }
    const int64_t most = (int64_t(1) << 31) / 257;
    if (a_bytes <= kMostCopied && b_bytes <= kMostCopied - a_bytes && (a_fits || ld_a * 2 < most) && (b_fits || ld_b * 2 < most)) {
        const LinearChoice *tiles = linear_tile_choices<KIND>(&count);
        look(tiles, count, true);
        if constexpr (KIND != kWgrad) {
            const LinearChoice *streams = linear_stream_choices<KIND>(&count);
            look(streams, count, true);
        }
    }
    return best;
}

// Rows of bf16 at any address to aligned ones, zeros behind their ends: eight values a thread.
struct Copy {
    const Bf16 *from;
    int64_t ld;
    Bf16 *to;
    int64_t rows, chunks;   // of eight values a row
    int cols;
};
constexpr int kCopyThreads = 256;
__global__ void __launch_bounds__(kCopyThreads) linear_copy_kernel(Copy a, Copy b, unsigned groups_a) {
    const bool first = blockIdx.x < groups_a;
    const Copy &c = first ? a : b;
    const int64_t id = (int64_t)(first ? blockIdx.x : blockIdx.x - groups_a) * kCopyThreads + threadIdx.x;
    const int64_t row = id / c.chunks, at = (id - row * c.chunks) * 8;
    if (row >= c.rows) return;
    const Raw8<Bf16> v = raw8(c.from + row * c.ld + at, c.cols - (int)at);
    __builtin_memcpy(__builtin_assume_aligned(c.to + row * c.chunks * 8 + at, 16), v.v, sizeof(v.v));
}

// The sums of the parts, in their order, and the epilogue: a row's kJoinEach columns a thread.  Bound by memory (4
// splits of 1024 x 2048 fp32 8.9 us, 4.7 TB/s); a launch of its own, since workgroups that waited for each other's sums
// would need memory cleared before every call.
constexpr int kJoinThreads = 256, kJoinEach = 4, kJoinAtOnce = 4;
template <typename T>
__global__ void __launch_bounds__(kJoinThreads) linear_join_kernel(LinearArgs p, int rows) {
    const int chunks = (p.N + kJoinEach - 1) / kJoinEach;
    const int64_t id = (int64_t)blockIdx.x * kJoinThreads + threadIdx.x;
    const int row = (int)(id / chunks), n = (int)(id - (int64_t)row * chunks) * kJoinEach;
    if (row >= rows) return;
    float v[kJoinEach] = {};
    for (int s0 = 0; s0 < p.splits; s0 += kJoinAtOnce) {
        float q[kJoinAtOnce][kJoinEach];
#pragma unroll
        for (int k = 0; k < kJoinAtOnce; ++k)
            Epilogue<T, kJoinEach>::load(p.part, 1, ((int64_t)(s0 + k < p.splits ? s0 + k : 0) * rows + row) * p.N + n, p.N - n, q[k]);
#pragma unroll
        for (int k = 0; k < kJoinAtOnce; ++k)
#pragma unroll
            for (int i = 0; i < kJoinEach; ++i) v[i] += s0 + k < p.splits ? q[k][i] : 0.f;
    }
    finish_at<T, kJoinEach>(p, row, n, v);
}

template <Kind KIND>
int64_t workspace(const LinearArgs &a) {
    const Plan w = plan<KIND>(a);
    return w.part_bytes + w.a_bytes + w.b_bytes;
}

template <Kind KIND>
xtc_status launch(const LinearArgs &given, void *workspace, int64_t bytes, hipStream_t s) {
    LinearArgs a = given;
    const Plan w = plan<KIND>(a);
    const int64_t need = w.part_bytes + w.a_bytes + w.b_bytes;
    if (need > bytes) return XTC_ERR_BAD_SHAPE;
    if (need > 0 && !workspace) return XTC_ERR_NULL_POINTER;
    unsigned char *ws = static_cast<unsigned char *>(workspace);
    a.splits = w.splits;
    a.k_each = w.k_each;
    a.part = reinterpret_cast<float *>(ws);
    if (w.copy_a || w.copy_b) {
        Copy ca = {}, cb = {};
        int64_t groups_a = 0, groups_b = 0;
        if (w.copy_a) {
            ca = Copy{static_cast<const Bf16 *>(a.A), a.lda, reinterpret_cast<Bf16 *>(ws + w.part_bytes), a.T, w.ld_a / 8, a.K};
            groups_a = cdiv(ca.rows * ca.chunks, kCopyThreads);
            a.A = ca.to;
            a.lda = w.ld_a;
        }
        if (w.copy_b) {
            cb = Copy{static_cast<const Bf16 *>(a.B), a.ldb, reinterpret_cast<Bf16 *>(ws + w.part_bytes + w.a_bytes),
                      KIND == kBf16T ? a.N : KIND == kWgrad ? a.T : a.K, w.ld_b / 8, KIND == kBf16T ? a.K : a.N};
            groups_b = cdiv(cb.rows * cb.chunks, kCopyThreads);
            a.B = cb.to;
            a.ldb = w.ld_b;
        }
        if (groups_a + groups_b >= kMostGroups) return XTC_ERR_TOO_LARGE;
        if (groups_a + groups_b > 0) {
            linear_copy_kernel<<<(unsigned)(groups_a + groups_b), kCopyThreads, 0, s>>>(ca, cb, (unsigned)groups_a);
            const xtc_status st = hip_status(hipGetLastError());
            if (st != XTC_OK) return st;
        }
    }
    const xtc_status st = w.choice->launch(a, s);
    if (st != XTC_OK || a.splits == 1) return st;
    const int64_t rows = KIND == kWgrad ? a.K : a.T;
    const int64_t groups = cdiv(rows * cdiv(a.N, kJoinEach), kJoinThreads);
    if (groups >= kMostGroups) return XTC_ERR_TOO_LARGE;
    const auto join = a.out_bf16 ? linear_join_kernel<__bf16> : linear_join_kernel<float>;
    join<<<(unsigned)groups, kJoinThreads, 0, s>>>(a, (int)rows);
    return hip_status(hipGetLastError());
}

// dz = dy act'(z), and the column sums of a slab of rows: LANES lanes take eight columns of a row each, the
// workgroup's teams of LANES rows in turn, kSlopeRows on their way together.  Of many rows a team is a wave.  Bound by memory:
// 8192 x 4096 bf16 (gelu_tanh) 37 to 40 us, 5 to 5.4 TB/s past the caches, and 4.5 for the join of 256 rows of sums (one row
// at a time through the caches 47).  About 25 vector instructions an element, two of them at a quarter of the rate,
// take half of that time beside the memory's.
// Of few rows 32 teams of eight lanes share a workgroup that has them all, and whose sums are the result: one launch (64 x
// 2816 bf16 5.0 us, 8.4 by two; 256 rows 8.0 and 8.4, in fp32 10.6 and 8.8).
// Four waves a SIMD, whatever the registers would allow: with five their loads find fewer lines together (8192 x 4096 in bf16,
// gelu_tanh, 43.0 us with four, 44.0 with five).
constexpr int kSlopeThreads = 256, kSlopeRows = 4;   // (rows on their way at once)
constexpr int kSlopeMany = 64, kSlopeFew = 8, kFewRows = 128;
template <typename TY, typename TZ, int LANES>
__global__ void __launch_bounds__(kSlopeThreads) __attribute__((amdgpu_waves_per_eu(4, 4))) activation_backward_kernel(ActivationArgs p) {
    constexpr int COLUMNS = LANES * 8, TEAMS = kSlopeThreads / LANES;
    __shared__ __attribute__((aligned(16))) float sums[TEAMS][COLUMNS];
    const int lane = threadIdx.x % LANES, team = threadIdx.x / LANES;
    const int c = blockIdx.x * COLUMNS + lane * 8, valid = p.N - c;
    float sum[8] = {0, 0, 0, 0, 0, 0, 0, 0};
    with_activation(p.act, [&](auto ACT) __attribute__((always_inline)) {
        const int64_t step = (int64_t)gridDim.y * TEAMS;
        for (int64_t t = (int64_t)blockIdx.y * TEAMS + team; t < p.T; t += kSlopeRows * step) {
            Raw8<TY> y[kSlopeRows];
            Raw8<TZ> z[kSlopeRows];
#pragma unroll
            for (int r = 0; r < kSlopeRows; ++r) {
                // (past the last row that one again: loads in a branch would wait for it)
                const int64_t at = t + r * step < p.T ? t + r * step : p.T - 1;
                y[r] = raw8_once(static_cast<const TY *>(p.DY) + at * p.lddy + c, valid);
                z[r] = raw8_once(static_cast<const TZ *>(p.Z) + at * p.ldz + c, valid);
            }
#pragma unroll
            for (int r = 0; r < kSlopeRows; ++r) {
                const int64_t at = t + r * step;
                float d[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    d[i] = y[r].at(i) * slope<ACT()>(z[r].at(i));
                    sum[i] += at < p.T ? d[i] : 0.f;
                }
                store8_to(static_cast<Bf16 *>(p.DZ) + at * p.lddz + c, at < p.T ? valid : 0, d, p.past);
            }
        }
    });
    if (!p.DB) return;
    __builtin_memcpy(__builtin_assume_aligned(&sums[team][lane * 8], 16), sum, sizeof(sum));
    __syncthreads();
    float *to = gridDim.y > 1 ? p.partial + (int64_t)blockIdx.y * p.N : p.DB;
    for (int q = threadIdx.x; q < COLUMNS; q += kSlopeThreads) {
        float s = 0.f;
#pragma unroll
        for (int w = 0; w < TEAMS; ++w) s += sums[w][q];
        if ((int)blockIdx.x * COLUMNS + q < p.N) to[blockIdx.x * COLUMNS + q] = s;
    }
}

}  // namespace

int64_t linear_workspace(const LinearArgs &a, bool b_rows_n) {
    return b_rows_n ? workspace<kBf16T>(a) : workspace<kBf16N>(a);
}
xtc_status launch_linear(const LinearArgs &a, bool b_rows_n, void *workspace, int64_t bytes, hipStream_t s) {
    return b_rows_n ? launch<kBf16T>(a, workspace, bytes, s) : launch<kBf16N>(a, workspace, bytes, s);
}
int64_t linear_wgrad_workspace(const LinearArgs &a) { return workspace<kWgrad>(a); }
xtc_status launch_linear_wgrad(const LinearArgs &a, void *workspace, int64_t bytes, hipStream_t s) {
    return launch<kWgrad>(a, workspace, bytes, s);
}

namespace {

template <Kind KIND>
int kernel_place(const LinearArgs &a, int *kernels, int *splits) {
    const Plan w = plan<KIND>(a);
    int count = 0;
    linear_tile_choices<KIND>(kernels);
    if constexpr (KIND != kWgrad) {
        linear_stream_choices<KIND>(&count);
        *kernels += count;
    }
    if (!(aligned_rows(a.A, a.lda) && aligned_rows(a.B, a.ldb) && (KIND == kWgrad || a.K % 8 == 0))) {
        linear_any_choices<KIND>(&count);
        *kernels += count;
    }
    *splits = w.splits;
    return w.place;
}

}  // namespace

int linear_kernel(const LinearArgs &a, int kind, int *kernels, int *splits) {
    return kind == kBf16N   ? kernel_place<kBf16N>(a, kernels, splits)
           : kind == kBf16T ? kernel_place<kBf16T>(a, kernels, splits)
                            : kernel_place<kWgrad>(a, kernels, splits);
}

int activation_slabs(int64_t T, int64_t N) {
    if (T <= kFewRows) return 1;
    // (a trip of kSlopeRows rows a team at least: 1024 x 4096 10.7 us, with one row a team 22)
    const int64_t across = cdiv(N, kSlopeMany * 8), rows = cdiv(T, kSlopeThreads / kSlopeMany * kSlopeRows), most = across < 2048 ? 2048 / across : 1;
    return (int)(rows < most ? rows : most);
}

namespace {

template <int LANES>
auto slope_kernel(const ActivationArgs &a) {
    return a.dy_f32 ? (a.z_f32 ? activation_backward_kernel<float, float, LANES> : activation_backward_kernel<float, Bf16, LANES>)
                    : (a.z_f32 ? activation_backward_kernel<Bf16, float, LANES> : activation_backward_kernel<Bf16, Bf16, LANES>);
}

}  // namespace

xtc_status launch_activation_backward(const ActivationArgs &given, hipStream_t s) {
    ActivationArgs a = given;
    a.past = whole_lines(a.DZ, a.lddz, 2);
    const int slabs = activation_slabs(a.T, a.N);
    // (64 columns a workgroup there: 2^30 of them would be 2^32 threads, which are no launch)
    const bool few = a.T <= kFewRows && a.N <= 1 << 29;
    const auto kernel = few ? slope_kernel<kSlopeFew>(a) : slope_kernel<kSlopeMany>(a);
    kernel<<<dim3((unsigned)cdiv(a.N, few ? kSlopeFew * 8 : kSlopeMany * 8), (unsigned)slabs), kSlopeThreads, 0, s>>>(a);
    const xtc_status st = hip_status(hipGetLastError());
    if (st != XTC_OK || !a.DB || slabs == 1) return st;
    return launch_column_sums(a.partial, slabs, a.N, a.DB, nullptr, s);
}

}  // namespace xtc

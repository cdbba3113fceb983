// The linear layer: the choice of its kernel and splits, the join of the splits' sums, and the
// gradients of its activation and bias.
#include "linear.h"

namespace xtc {
namespace {

bool aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }

// As for the grouped products: 16-byte aligned rows, whole 16-byte chunks of k where they
// run along it, strides that keep the offsets within a tile in 31 bits.
template <Kind KIND>
bool aligned_rows(const LinearArgs &a) {
    const int64_t most = (int64_t(1) << 31) / 257;
    if (!aligned16(a.A) || !aligned16(a.B) || a.lda * 2 % 16 || a.ldb * 2 % 16) return false;
    if (KIND != kWgrad && a.K * 2 % 16) return false;
    return a.lda * 2 < most && a.ldb * 2 < most;
}

// A kernel and the parts of the reduction it is launched with.
struct Plan {
    const Choice *choice;     // null: the kernel for rows at any address
    int splits, k_each;
    int place;
};

constexpr int kSplitStep = 128;      // parts of the reduction are whole stages of every kernel

// Microseconds of a launch over `splits` parts: rounds of tiles on 256 CUs as for the
// grouped products, and the way of the parts' sums to memory and back.
double estimate_us(const Choice &c, int64_t rows, int64_t cols, int64_t reduce, int64_t weights, int splits, int64_t k_each) {
    const double stages = (double)cdiv(k_each < reduce ? k_each : reduce, 64), slots = 256. * c.per_cu;
    const int64_t n = cdiv(rows, c.bm) * cdiv(cols, c.bn) * splits, whole = (int64_t)(n / slots);
    const double rest = n - whole * slots;
    const int64_t held = cdiv((int64_t)rest, 256);
    const bool from_memory = weights * 2 > 64e6;
    const double one = from_memory ? c.cold : c.one, full = c.per_cu > 1 ? c.full : one;
    double us = whole * (stages * full + c.fixed);
    if (held > 0) {
        const double last = stages * (held > 1 ? one + (full - one) * (held - 1) / (c.per_cu - 1) : one) + c.fixed;
        us += whole > 0 && c.per_cu > 1 ? last / 2 : last;
    }
    if (splits > 1) us += 3 + 8. * splits * rows * cols / 4e6;
    return us;
}

template <Kind KIND>
Plan plan(const LinearArgs &a) {
    const int64_t rows = KIND == kWgrad ? a.K : a.T, reduce = KIND == kWgrad ? a.T : a.K;
    const int64_t whole = cdiv(reduce > 1 ? reduce : 1, kSplitStep) * kSplitStep;
    Plan best = {nullptr, 1, (int)whole, -1};
    if (!aligned_rows<KIND>(a)) return best;
    double least = 0;
    int seen = 0;
    auto look = [&](const Choice *c, int count) {
        for (int i = 0; i < count; ++i, ++seen)
            for (int want = 1; want <= 16; want *= 2) {
                const int64_t each = cdiv(cdiv(reduce > 1 ? reduce : 1, want), kSplitStep) * kSplitStep;
                const int splits = (int)cdiv(reduce > 1 ? reduce : 1, each);
                if (want > 1 && (splits < 2 || each < 512)) break;
                const double us = estimate_us(c[i], rows, a.N, reduce, (int64_t)a.N * a.K, splits, each);
                if (!best.choice || us < least) {
                    best = Plan{&c[i], splits, (int)each, seen};
                    least = us;
                }
            }
    };
    int count = 0;
    const Choice *tiles = linear_tile_choices<KIND>(&count);
    look(tiles, count);
    if constexpr (KIND != kWgrad) {
        const Choice *streams = linear_stream_choices<KIND>(&count);
        look(streams, count);
    }
    return best;
}

// The sums of the parts, in their order, and the epilogue: a row's EACH columns a thread.
constexpr int kJoinThreads = 256, kJoinEach = 4;
template <typename T>
__global__ void __launch_bounds__(kJoinThreads) linear_join_kernel(LinearArgs p, int rows) {
    const int chunks = (p.N + kJoinEach - 1) / kJoinEach;
    const int64_t id = (int64_t)blockIdx.x * kJoinThreads + threadIdx.x;
    const int row = (int)(id / chunks), n = (int)(id - (int64_t)row * chunks) * kJoinEach;
    if (row >= rows) return;
    float v[kJoinEach] = {};
    for (int s = 0; s < p.splits; ++s) {
        float q[kJoinEach];
        Epilogue<T, kJoinEach>::load(p.part, 1, ((int64_t)s * rows + row) * p.N + n, p.N - n, q);
#pragma unroll
        for (int i = 0; i < kJoinEach; ++i) v[i] += q[i];
    }
    finish_at<T, kJoinEach>(p, row, n, v);
}

template <Kind KIND>
int64_t workspace(const LinearArgs &a) {
    const Plan w = plan<KIND>(a);
    return w.splits > 1 ? 4 * (int64_t)w.splits * (KIND == kWgrad ? a.K : a.T) * a.N : 0;
}

template <Kind KIND>
xtc_status launch(const LinearArgs &given, hipStream_t s) {
    LinearArgs a = given;
    const Plan w = plan<KIND>(a);
    a.splits = w.splits;
    a.k_each = w.k_each;
    if (!w.choice) return launch_linear_any<KIND>(a, s);
    const xtc_status st = w.choice->launch(a, s);
    if (st != XTC_OK || a.splits == 1) return st;
    const int64_t rows = KIND == kWgrad ? a.K : a.T;
    const int64_t groups = cdiv(rows * cdiv(a.N, kJoinEach), kJoinThreads);
    if (groups >= kMostGroups) return XTC_ERR_TOO_LARGE;
    const auto join = a.out_bf16 ? linear_join_kernel<__bf16> : linear_join_kernel<float>;
    join<<<(unsigned)groups, kJoinThreads, 0, s>>>(a, (int)rows);
    return hip_status(hipGetLastError());
}

// dz = dy act'(z), and the column sums of a slab of rows: a wave takes 512 columns of a row at
// a time, eight a lane, the workgroup's four waves rows in turn.
constexpr int kSlopeColumns = 512, kSlopeWaves = 4;
template <typename TY, typename TZ>
__global__ void __launch_bounds__(kSlopeWaves * 64) activation_backward_kernel(ActivationArgs p) {
    __shared__ float sums[kSlopeWaves - 1][8][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int c = blockIdx.x * kSlopeColumns + lane * 8, valid = p.N - c;
    float sum[8] = {0, 0, 0, 0, 0, 0, 0, 0};
    with_activation(p.act, [&](auto ACT) __attribute__((always_inline)) {
        const int64_t step = (int64_t)gridDim.y * kSlopeWaves;
        for (int64_t t = (int64_t)blockIdx.y * kSlopeWaves + wave; t < p.T; t += step) {
            float d[8], z[8];
            load8(static_cast<const TY *>(p.DY) + t * p.lddy + c, valid, d);
            load8(static_cast<const TZ *>(p.Z) + t * p.ldz + c, valid, z);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                d[i] *= slope<ACT()>(z[i]);
                sum[i] += d[i];
            }
            store8(static_cast<Bf16 *>(p.DZ) + t * p.lddz + c, valid, d);
        }
    });
    if (!p.DB) return;
    if (wave > 0) {
#pragma unroll
        for (int i = 0; i < 8; ++i) sums[wave - 1][i][lane] = sum[i];
    }
    __syncthreads();
    if (wave > 0) return;
#pragma unroll
    for (int i = 0; i < 8; ++i)
#pragma unroll
        for (int w = 0; w < kSlopeWaves - 1; ++w) sum[i] += sums[w][i][lane];
    store8(p.partial + (int64_t)blockIdx.y * p.N + c, valid, sum);
}

}  // namespace

int64_t linear_workspace(const LinearArgs &a, bool b_rows_n) {
    return b_rows_n ? workspace<kBf16T>(a) : workspace<kBf16N>(a);
}
xtc_status launch_linear(const LinearArgs &a, bool b_rows_n, hipStream_t s) {
    return b_rows_n ? launch<kBf16T>(a, s) : launch<kBf16N>(a, s);
}
int64_t linear_wgrad_workspace(const LinearArgs &a) { return workspace<kWgrad>(a); }
xtc_status launch_linear_wgrad(const LinearArgs &a, hipStream_t s) { return launch<kWgrad>(a, s); }

int activation_slabs(int64_t T, int64_t N) {
    const int64_t across = cdiv(N, kSlopeColumns), rows = cdiv(T, kSlopeWaves), most = across < 2048 ? 2048 / across : 1;
    return (int)(rows < most ? (rows > 1 ? rows : 1) : most);
}

xtc_status launch_activation_backward(const ActivationArgs &a, hipStream_t s) {
    const int slabs = activation_slabs(a.T, a.N);
    const auto kernel = a.dy_f32 ? (a.z_f32 ? activation_backward_kernel<float, float> : activation_backward_kernel<float, Bf16>)
                                 : (a.z_f32 ? activation_backward_kernel<Bf16, float> : activation_backward_kernel<Bf16, Bf16>);
    kernel<<<dim3((unsigned)cdiv(a.N, kSlopeColumns), (unsigned)slabs), kSlopeWaves * 64, 0, s>>>(a);
    const xtc_status st = hip_status(hipGetLastError());
    if (st != XTC_OK || !a.DB) return st;
    return launch_column_sums(a.partial, slabs, a.N, a.DB, nullptr, s);
}

}  // namespace xtc

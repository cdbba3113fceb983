// The rows of a mixture's experts back at their tokens:
//
//   out_t = residual_t + sum_j p_tj rows[row_tj],
//
// and the gradients drows[row_tj] = p_tj dout_t, dp_tj = <dout_t, rows[row_tj]>; sums are fp32, over j in
// its order.  Rows outside the array (-1: a choice that was masked) count as nothing.
#include "operators.h"
#include "values.h"

namespace xtc {
namespace {

constexpr int kWaves = 4, kColumns = 512;      // columns of a wave, eight a lane

__device__ __forceinline__ int wave_id() { return __builtin_amdgcn_readfirstlane(threadIdx.x >> 6); }

// A wave a token and 512 columns of it: kAtOnce rows are on their way together.  Bound by memory: 4096 tokens of eight
// rows of 2048 bf16 with a residual 28 us, 6.0 TB/s with what the last-level cache serves (45 us with loads that keep
// their lines in L2, where no other token finds them).
constexpr int kAtOnce = 8;
template <typename T, typename R, typename O>
__global__ void __launch_bounds__(kWaves * 64) combine_kernel(CombineArgs p, int chunks) {
    const int64_t id = (int64_t)blockIdx.x * kWaves + wave_id(), t = id / chunks;
    if (t >= p.T) return;
    const int c = (int)(id - t * chunks) * kColumns + (threadIdx.x & 63) * 8, valid = p.D - c;
    float sum[8] = {0, 0, 0, 0, 0, 0, 0, 0};
    if (p.RES) load8(static_cast<const R *>(p.RES) + t * p.ldr + c, valid, sum);
    for (int j0 = 0; j0 < p.top; j0 += kAtOnce) {
        Raw8<T> v[kAtOnce];
        float w[kAtOnce];
#pragma unroll
        for (int j = 0; j < kAtOnce; ++j) {
            int64_t r = -1;
            w[j] = 1.f;
            if (j0 + j < p.top) {
                r = p.row[t * p.top + j0 + j];
                if (p.P) w[j] = p.P[t * p.top + j0 + j];
            }
            const bool in = r >= 0 && r < p.R;
            w[j] = in ? w[j] : 0.f;
            v[j] = raw8_once(static_cast<const T *>(p.rows) + (in ? r : 0) * p.ldrows + c, in ? valid : 0);
        }
#pragma unroll
        for (int j = 0; j < kAtOnce; ++j)
#pragma unroll
            for (int i = 0; i < 8; ++i) sum[i] += w[j] * v[j].at(i);
    }
    store8(static_cast<O *>(p.out) + t * p.ldo + c, valid, sum);
}

// SHARE waves a token, 512 columns each in turn: their part of dout's row stays in registers over the
// rows of up to kAtOnce choices, and their sums of dp meet in LDS.  Bound by memory: 4095 tokens of eight rows of 2048
// bf16 61 us, 4.7 TB/s of its 286 MB past the caches (a wave a token, through the caches, 120).
template <typename T, typename G, int SHARE>
__global__ void __launch_bounds__(kWaves * 64) combine_backward_kernel(CombineBackwardArgs p) {
    __shared__ float part[kWaves][kAtOnce];
    const int wave = wave_id(), lane = threadIdx.x & 63, share = wave % SHARE;
    const int64_t t = (int64_t)blockIdx.x * (kWaves / SHARE) + wave / SHARE;
    if (t >= p.T) return;                // (SHARE > 1: the whole workgroup)
    for (int j0 = 0; j0 < p.top; j0 += kAtOnce) {
        float w[kAtOnce], dot[kAtOnce];
        int64_t r[kAtOnce];
#pragma unroll
        for (int j = 0; j < kAtOnce; ++j) {
            r[j] = j0 + j < p.top ? p.row[t * p.top + j0 + j] : -1;
            if (r[j] >= p.R) r[j] = -1;
            w[j] = r[j] >= 0 ? p.P[t * p.top + j0 + j] : 0.f;
            dot[j] = 0.f;
        }
        for (int c = share * kColumns + lane * 8; c < p.D; c += SHARE * kColumns) {
            const int valid = p.D - c;
            float d[8];
            Raw8<T> v[kAtOnce];
#pragma unroll
            for (int j = 0; j < kAtOnce; ++j)
                v[j] = raw8_once(static_cast<const T *>(p.rows) + (r[j] >= 0 ? r[j] : 0) * p.ldrows + c, r[j] >= 0 ? valid : 0);
            load8(static_cast<const G *>(p.DOUT) + t * p.lddo + c, valid, d);
#pragma unroll
            for (int j = 0; j < kAtOnce; ++j) {
                if (r[j] < 0) continue;
                float o[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    dot[j] += d[i] * v[j].at(i);
                    o[i] = w[j] * d[i];
                }
                store8_to(static_cast<T *>(p.DROWS) + r[j] * p.lddr + c, valid, o, p.past);
            }
        }
        if constexpr (SHARE > 1) {
            if (j0 > 0) __syncthreads();
#pragma unroll
            for (int j = 0; j < kAtOnce; ++j) {
                const float s = lanes_sum<64>(dot[j]);
                if (lane == j) part[wave][j] = s;
            }
            __syncthreads();
            if (wave == 0 && lane < kAtOnce && j0 + lane < p.top) {
                float s = 0.f;
#pragma unroll
                for (int i = 0; i < SHARE; ++i) s += part[i][lane];
                p.DP[t * p.top + j0 + lane] = s;
            }
        } else {
#pragma unroll
            for (int j = 0; j < kAtOnce; ++j) {
                const float s = lanes_sum<64>(dot[j]);
                if (lane == 0 && j0 + j < p.top) p.DP[t * p.top + j0 + j] = s;
            }
        }
    }
    // this token's share of the rows that belong to none: zeros
    for (int j = 0; j < p.top; ++j) {
        const int64_t i = t * p.top + j;
        if (i >= p.R || p.token[i] >= 0) continue;
        const float zero[8] = {0, 0, 0, 0, 0, 0, 0, 0};
        for (int c = share * kColumns + lane * 8; c < p.D; c += SHARE * kColumns)
            store8_to(static_cast<T *>(p.DROWS) + i * p.lddr + c, p.D - c, zero, p.past);
    }
}

template <typename T, typename R>
auto pick(xtc_dtype out_dtype) { return out_dtype == XTC_F32 ? combine_kernel<T, R, float> : combine_kernel<T, R, Bf16>; }

}  // namespace

xtc_status launch_combine(const CombineArgs &a, xtc_dtype dtype, xtc_dtype r_dtype, xtc_dtype out_dtype, hipStream_t s) {
    const int64_t chunks = (a.D + kColumns - 1) / kColumns, groups = (a.T * chunks + kWaves - 1) / kWaves;
    if (groups >= kMostGroups) return XTC_ERR_TOO_LARGE;
    const auto kernel = dtype == XTC_F32 ? (r_dtype == XTC_F32 ? pick<float, float>(out_dtype) : pick<float, Bf16>(out_dtype))
                                         : (r_dtype == XTC_F32 ? pick<Bf16, float>(out_dtype) : pick<Bf16, Bf16>(out_dtype));
    kernel<<<(unsigned)groups, kWaves * 64, 0, s>>>(a, (int)chunks);
    return hip_status(hipGetLastError());
}

namespace {

template <int SHARE>
xtc_status launch_shared(const CombineBackwardArgs &a, xtc_dtype dtype, xtc_dtype g_dtype, hipStream_t s) {
    const int64_t each = kWaves / SHARE, groups = (a.T + each - 1) / each;
    if (groups >= kMostGroups) return XTC_ERR_TOO_LARGE;
    const auto kernel = dtype == XTC_F32 ? (g_dtype == XTC_F32 ? combine_backward_kernel<float, float, SHARE> : combine_backward_kernel<float, Bf16, SHARE>)
                                         : (g_dtype == XTC_F32 ? combine_backward_kernel<Bf16, float, SHARE> : combine_backward_kernel<Bf16, Bf16, SHARE>);
    kernel<<<(unsigned)groups, kWaves * 64, 0, s>>>(a);
    return hip_status(hipGetLastError());
}

}  // namespace

xtc_status launch_combine_backward(const CombineBackwardArgs &given, xtc_dtype dtype, xtc_dtype g_dtype, hipStream_t s) {
    CombineBackwardArgs a = given;
    a.past = whole_lines(a.DROWS, a.lddr, dtype == XTC_F32 ? 4 : 2);
    return a.D > kColumns ? launch_shared<kWaves>(a, dtype, g_dtype, s) : launch_shared<1>(a, dtype, g_dtype, s);
}

}  // namespace xtc

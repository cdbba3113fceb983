// Root-mean-square norm with the residual's addition, its gradient, and the
// conversion of rows and blocks to e4m3 with a scale.
//
//   h = x + r, rstd = 1 / sqrt(mean_j h_j^2 + eps), y_j = w_j h_j rstd
//
// with h and every sum in fp32.  In 8 bits the 128 values of a block share
// s = max(amax / 448, 2^-126) and are rounded from y / s.
//
// The gradient, with xh = h rstd and g = dy w:
//   dx = rstd (g - xh mean_j(g_j xh_j)) + dr,   dw_j = sum_t dy_tj xh_tj
#include <type_traits>

#include "operators.h"
#include "values.h"

namespace xtc {
namespace {

constexpr int kThreads = 256;
constexpr int kStep = kThreads * 8;     // columns that a workgroup covers at once

// Sum of v over the workgroup, in every thread.
__device__ __forceinline__ float group_sum(float v, float *scratch) {
    v = lanes_sum<64>(v);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) scratch[threadIdx.x >> 6] = v;
    __syncthreads();
    float s = scratch[0];
#pragma unroll
    for (int i = 1; i < kThreads / 64; ++i) s += scratch[i];
    return s;
}

__device__ __forceinline__ void load_weight(const void *w, int w_f32, const float *, int c, int valid, float (&v)[8]) {
    load8(static_cast<const float *>(w) + c, valid, v);
}
__device__ __forceinline__ void load_weight(const void *w, int w_f32, const Bf16 *, int c, int valid, float (&v)[8]) {
    if (w_f32) load8(static_cast<const float *>(w) + c, valid, v);
    else load8(static_cast<const Bf16 *>(w) + c, valid, v);
}

__device__ __forceinline__ Raw8<float> raw_weight(const void *w, int, const float *, int c, int valid) {
    return raw8(static_cast<const float *>(w) + c, valid);
}
// (as fp32 whichever type it has)
__device__ __forceinline__ Raw8<float> raw_weight(const void *w, int w_f32, const Bf16 *, int c, int valid) {
    if (w_f32) return raw8(static_cast<const float *>(w) + c, valid);
    const Raw8<Bf16> b = raw8(static_cast<const Bf16 *>(w) + c, valid);
    Raw8<float> r;
#pragma unroll
    for (int i = 0; i < 8; ++i) r.v[i] = b.at(i);
    return r;
}

// NT threads share a row and hold it in registers, NV groups of eight columns
// each, between the sum of squares and the outputs: every row is read once.
// A workgroup has 256 threads or NT.  8192 x 4096 bf16 with a residual to 8
// bits, bound by memory: 52 us, 4.5 TB/s of its 236 MB where a copy reaches 5.3
// (the loop kernel below, which reads a row twice, 67).  One row of 4096 columns
// takes 3.9 us, the time of a launch and two trips to memory.
template <int NT>
struct RowTeam {
    static constexpr int THREADS = NT > 256 ? NT : 256, ROWS = THREADS / NT;
    // Sum over the row's threads, in each of them.
    static __device__ __forceinline__ float sum(float v, float *scratch) {
        v = lanes_sum<64>(v);
        if constexpr (NT > 64) {
            __syncthreads();
            if ((threadIdx.x & 63) == 0) scratch[threadIdx.x >> 6] = v;
            __syncthreads();
            v = 0.f;
#pragma unroll
            for (int i = 0; i < NT / 64; ++i) v += scratch[i];
        }
        return v;
    }
};

template <typename T, bool QUANT, int NT, int NV>
__global__ void __launch_bounds__(RowTeam<NT>::THREADS) rmsnorm_kernel(NormArgs p) {
    typedef RowTeam<NT> Team;
    __shared__ float scratch[NT / 64];
    const int tid = threadIdx.x % NT, D = p.D;
    // (a whole team past the last row leaves; with more than one wave it has the workgroup to itself)
    const int64_t t = (int64_t)blockIdx.x * Team::ROWS + threadIdx.x / NT;
    if (t >= p.T) return;
    const T *x = static_cast<const T *>(p.X) + t * p.ldx;
    const T *r = p.R ? static_cast<const T *>(p.R) + t * p.ldr : nullptr;
    Raw8<T> rx[NV], rr[NV];
#pragma unroll
    for (int v = 0; v < NV; ++v) {
        const int c = (v * NT + tid) * 8;
        rx[v] = raw8(x + c, D - c);
        if (r) rr[v] = raw8(r + c, D - c);
    }
    float h[NV][8], sum = 0.f;
#pragma unroll
    for (int v = 0; v < NV; ++v)
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            h[v][i] = r ? rx[v].at(i) + rr[v].at(i) : rx[v].at(i);
            sum += h[v][i] * h[v][i];
        }
    sum = Team::sum(sum, scratch);
    const float rstd = 1.f / sqrtf(sum / (float)D + p.eps);
    if (tid == 0 && p.rstd) p.rstd[t] = rstd;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
        const int c = (v * NT + tid) * 8, valid = D - c;
        const Raw8<float> w = raw_weight(p.W, p.w_f32, x, c, valid);
        if (p.H) store8(static_cast<T *>(p.H) + t * p.ldh + c, valid, h[v]);
        float y[8], amax = 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            y[i] = h[v][i] * rstd * w.v[i];
            if constexpr (QUANT) amax = fmaxf(amax, finite_abs(y[i]));
        }
        if constexpr (QUANT) {
            const float s = fp8_scale(lanes_max<16>(amax));
            store_fp8(static_cast<uint8_t *>(p.Y) + t * p.ldy + c, valid, to_fp8(y, s));
            if ((tid & 15) == 0 && valid > 0) p.S[t * p.lds + c / kScaleBlock] = s;
        } else {
            store8(static_cast<T *>(p.Y) + t * p.ldy + c, valid, y);
        }
    }
}

// A workgroup per row, any number of columns: one pass for the sum of
// squares, another that reads the row again.
template <typename T, bool QUANT>
__global__ void __launch_bounds__(kThreads) rmsnorm_loop_kernel(NormArgs p) {
    __shared__ float scratch[kThreads / 64];
    const int tid = threadIdx.x, D = p.D;
    for (int64_t t = blockIdx.x; t < p.T; t += gridDim.x) {
        const T *x = static_cast<const T *>(p.X) + t * p.ldx;
        const T *r = p.R ? static_cast<const T *>(p.R) + t * p.ldr : nullptr;
        auto load_h = [&](int c, float (&h)[8]) {
            load8(x + c, D - c, h);
            if (r) {
                float q[8];
                load8(r + c, D - c, q);
#pragma unroll
                for (int i = 0; i < 8; ++i) h[i] += q[i];
            }
        };
        float sum = 0.f;
        for (int c = tid * 8; c < D; c += kStep) {
            float h[8];
            load_h(c, h);
#pragma unroll
            for (int i = 0; i < 8; ++i) sum += h[i] * h[i];
        }
        sum = group_sum(sum, scratch);
        const float rstd = 1.f / sqrtf(sum / (float)D + p.eps);
        if (tid == 0 && p.rstd) p.rstd[t] = rstd;
        // (whole trips: the lanes that share a block's scale stay together)
        for (int c0 = 0; c0 < D; c0 += kStep) {
            const int c = c0 + tid * 8, valid = D - c;
            float h[8], w[8], y[8];
            load_h(c, h);
            load_weight(p.W, p.w_f32, x, c, valid, w);
            if (p.H) store8(static_cast<T *>(p.H) + t * p.ldh + c, valid, h);
#pragma unroll
            for (int i = 0; i < 8; ++i) y[i] = h[i] * rstd * w[i];
            if constexpr (QUANT) {
                float amax = 0.f;
#pragma unroll
                for (int i = 0; i < 8; ++i) amax = fmaxf(amax, finite_abs(y[i]));
                const float s = fp8_scale(lanes_max<16>(amax));
                store_fp8(static_cast<uint8_t *>(p.Y) + t * p.ldy + c, valid, to_fp8(y, s));
                if ((tid & 15) == 0 && valid > 0) p.S[t * p.lds + c / kScaleBlock] = s;
            } else {
                store8(static_cast<T *>(p.Y) + t * p.ldy + c, valid, y);
            }
        }
    }
}

// The gradient in one pass: team by team, rows t, t + teams, ...; a thread keeps
// the sums over its rows of its columns' part of DW, and the workgroup leaves
// one row of partial sums.  The next row is on its way while one is computed.
// 8191 x 2048 bf16, bound by memory: 28.6 us, 4.7 TB/s; DX and DW by kernels of
// their own, which read the rows twice, took 151 us.
template <typename T, int NT, int NV>
__global__ void __launch_bounds__(RowTeam<NT>::THREADS) rmsnorm_backward_kernel(NormBackwardArgs p) {
    typedef RowTeam<NT> Team;
    __shared__ float scratch[NT / 64];
    __shared__ float sums[NT == 64 ? 3 * 64 * NV * 8 : 1];   // of the workgroup's other teams
    const int tid = threadIdx.x % NT, team = threadIdx.x / NT, D = p.D;
    const int64_t step = (int64_t)gridDim.x * Team::ROWS;
    Raw8<T> rx[NV], ry[NV], rr[NV];
    float w[NV][8], dw[NV][8], rstd_next = 0.f;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
        const int c = (v * NT + tid) * 8;
        const Raw8<float> q = raw_weight(p.W, p.w_f32, static_cast<const T *>(nullptr), c, D - c);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            w[v][i] = q.v[i];
            dw[v][i] = 0.f;
        }
    }
    auto fetch = [&](int64_t t) {
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            const int c = (v * NT + tid) * 8, valid = t < p.T ? D - c : 0;
            rx[v] = raw8(static_cast<const T *>(p.X) + t * p.ldx + c, valid);
            ry[v] = raw8(static_cast<const T *>(p.DY) + t * p.lddy + c, valid);
            if (p.DR) rr[v] = raw8(static_cast<const T *>(p.DR) + t * p.lddr + c, valid);
        }
        rstd_next = t < p.T ? p.rstd[t] : 0.f;
    };
    // (every team of a workgroup takes part in every trip: the sums below have barriers)
    int64_t t = (int64_t)blockIdx.x * Team::ROWS + team;
    fetch(t);
    for (int64_t t0 = (int64_t)blockIdx.x * Team::ROWS; t0 < p.T; t0 += step, t += step) {
        const float rstd = rstd_next;
        float h[NV][8], g[NV][8], d[NV][8], sum = 0.f;
#pragma unroll
        for (int v = 0; v < NV; ++v)
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                h[v][i] = rx[v].at(i) * rstd;
                const float y = ry[v].at(i);
                dw[v][i] += y * h[v][i];
                g[v][i] = y * w[v][i];
                d[v][i] = p.DR ? rr[v].at(i) : 0.f;
                sum += g[v][i] * h[v][i];
            }
        fetch(t + step);
        const float mean = Team::sum(sum, scratch) / (float)D;
        if (t < p.T) {
#pragma unroll
            for (int v = 0; v < NV; ++v) {
                const int c = (v * NT + tid) * 8;
                float o[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) o[i] = d[v][i] + rstd * (g[v][i] - h[v][i] * mean);
                store8(static_cast<T *>(p.DX) + t * p.lddx + c, D - c, o);
            }
        }
    }
    if constexpr (NT == 64) {
        if (team > 0) {
#pragma unroll
            for (int v = 0; v < NV; ++v)
#pragma unroll
                for (int i = 0; i < 8; ++i) sums[((team - 1) * NV * 8 + v * 8 + i) * 64 + tid] = dw[v][i];
        }
        __syncthreads();
        if (team > 0) return;
#pragma unroll
        for (int v = 0; v < NV; ++v)
#pragma unroll
            for (int i = 0; i < 8; ++i)
#pragma unroll
                for (int q = 0; q < 3; ++q) dw[v][i] += sums[(q * NV * 8 + v * 8 + i) * 64 + tid];
    }
#pragma unroll
    for (int v = 0; v < NV; ++v) {
        const int c = (v * NT + tid) * 8;
        store8(p.partial + (int64_t)blockIdx.x * D + c, D - c, dw[v]);
    }
}

// Rows of more columns than registers hold: DX and DW by kernels of their own, which
// read X and DY three times in all (4096 x 16384 bf16: 311 us, 1.7 TB/s of what one
// pass would move; 4096 x 8192 in one pass 64 us, 4.2 TB/s).
template <typename T>
__global__ void __launch_bounds__(kThreads) rmsnorm_dx_kernel(NormBackwardArgs p) {
    __shared__ float scratch[kThreads / 64];
    const int tid = threadIdx.x, D = p.D;
    for (int64_t t = blockIdx.x; t < p.T; t += gridDim.x) {
        const T *x = static_cast<const T *>(p.X) + t * p.ldx;
        const T *dy = static_cast<const T *>(p.DY) + t * p.lddy;
        const float rstd = p.rstd[t];
        float sum = 0.f;
        for (int c = tid * 8; c < D; c += kStep) {
            float h[8], g[8], w[8];
            load8(x + c, D - c, h);
            load8(dy + c, D - c, g);
            load_weight(p.W, p.w_f32, x, c, D - c, w);
#pragma unroll
            for (int i = 0; i < 8; ++i) sum += (g[i] * w[i]) * (h[i] * rstd);
        }
        const float mean = group_sum(sum, scratch) / (float)D;
        for (int c = tid * 8; c < D; c += kStep) {
            float h[8], g[8], w[8], d[8];
            load8(x + c, D - c, h);
            load8(dy + c, D - c, g);
            load_weight(p.W, p.w_f32, x, c, D - c, w);
            if (p.DR) load8(static_cast<const T *>(p.DR) + t * p.lddr + c, D - c, d);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float v = rstd * (g[i] * w[i] - h[i] * rstd * mean);
                d[i] = p.DR ? d[i] + v : v;
            }
            store8(static_cast<T *>(p.DX) + t * p.lddx + c, D - c, d);
        }
    }
}

// Sums of dy * xh over the slab blockIdx.y of rows.
template <typename T>
__global__ void __launch_bounds__(kThreads) rmsnorm_dw_kernel(NormBackwardArgs p) {
    const int c = (blockIdx.x * kThreads + threadIdx.x) * 8, valid = p.D - c;
    if (valid <= 0) return;
    float sum[8] = {0, 0, 0, 0, 0, 0, 0, 0};
    for (int64_t t = blockIdx.y; t < p.T; t += gridDim.y) {
        float h[8], g[8];
        load8(static_cast<const T *>(p.X) + t * p.ldx + c, valid, h);
        load8(static_cast<const T *>(p.DY) + t * p.lddy + c, valid, g);
        const float rstd = p.rstd[t];
#pragma unroll
        for (int i = 0; i < 8; ++i) sum[i] += g[i] * (h[i] * rstd);
    }
    store8(p.partial + (int64_t)blockIdx.y * p.D + c, valid, sum);
}

// Column sums of the slabs: sixteen columns a workgroup, 64 runs of slabs, each
// in its order, joined by halves (1024 rows of 2048 sums: 5 us, a few trips to
// memory and as many barriers).
constexpr int kJoinColumns = 16, kJoinThreads = 1024;
__global__ void __launch_bounds__(kJoinThreads) rmsnorm_dw_join_kernel(const float *partial, int slabs, int D, float *DW) {
    __shared__ float s[kJoinThreads];
    const int c = blockIdx.x * kJoinColumns + threadIdx.x % kJoinColumns, run = threadIdx.x / kJoinColumns;
    constexpr int RUNS = kJoinThreads / kJoinColumns;
    float sum = 0.f;
    if (c < D) {
#pragma unroll 8
        for (int g = run; g < slabs; g += RUNS) sum += partial[(int64_t)g * D + c];
    }
    s[threadIdx.x] = sum;
#pragma unroll
    for (int half = RUNS / 2; half > 0; half /= 2) {
        __syncthreads();
        if (run < half) s[threadIdx.x] += s[threadIdx.x + half * kJoinColumns];
    }
    if (run == 0 && c < D) DW[c] = s[threadIdx.x];
}

// e4m3 with a scale per 1 x 128 block: sixteen lanes a block.  Bound by memory:
// 4096 x 4096 bf16 in 11.2 us, 4.5 TB/s.
template <typename T>
__global__ void __launch_bounds__(kThreads) quantize_rows_kernel(QuantArgs p) {
    const int64_t kb = (p.K + kScaleBlock - 1) / kScaleBlock, blocks = p.M * kb;
    const int sub = threadIdx.x & 15;
    // (whole trips: every lane of a block takes part in its maximum)
    for (int64_t b = (int64_t)blockIdx.x * (kThreads / 16) + (threadIdx.x >> 4); b < blocks;
         b += (int64_t)gridDim.x * (kThreads / 16)) {
        const int64_t m = b / kb, k = (b - m * kb) * kScaleBlock + sub * 8;
        const int valid = (int)(p.K - k < 8 ? p.K - k : 8);
        float v[8];
        load8(static_cast<const T *>(p.X) + m * p.ldx + k, valid, v);
        float amax = 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) amax = fmaxf(amax, finite_abs(v[i]));
        const float s = fp8_scale(lanes_max<16>(amax));
        store_fp8(p.Q + m * p.ldq + k, valid, to_fp8(v, s));
        if (sub == 0) p.S[m * p.lds + (b - m * kb)] = s;
    }
}

// e4m3 with a scale per 128 x 128 block: a workgroup a block, which stays in
// registers between its maximum and its rounding.  Bound by memory: 8192 x 3001
// bf16, whose rows begin at odd addresses, in 17.6 us, 4.2 TB/s.
template <typename T>
__global__ void __launch_bounds__(kThreads) quantize_blocks_kernel(QuantArgs p) {
    __shared__ float scratch[kThreads / 64];
    // Workgroups go to the 8 XCDs in turn; each XCD gets a run of neighbouring blocks,
    // which share lines where rows do not begin on one (8192x3001: 22 us without, 17.6).
    const int xcd = (int)blockIdx.x & 7, each = (int)gridDim.x >> 3, rem = (int)gridDim.x & 7;
    const int64_t id = xcd * each + (xcd < rem ? xcd : rem) + ((int)blockIdx.x >> 3);
    const int64_t kb = (p.K + kScaleBlock - 1) / kScaleBlock, mb = id / kb, b = id - mb * kb;
    const int64_t k = b * kScaleBlock + (threadIdx.x & 15) * 8, m = mb * 128 + (threadIdx.x >> 4);
    const T *x = static_cast<const T *>(p.X) + m * p.ldx + k;
    uint8_t *q8 = p.Q + m * p.ldq + k;
    // rows 16 apart; one test for a whole block, whose loads then all go out together
    const bool whole = mb * 128 + 128 <= p.M && (b + 1) * kScaleBlock <= p.K;
    const int cols = p.K - k < 8 ? (int)(p.K - k) : 8, rows = (int)((p.M - m + 15) / 16 < 8 ? (p.M - m + 15) / 16 : 8);
    Raw8<T> r[8];
    if (whole) {
#pragma unroll
        for (int q = 0; q < 8; ++q) __builtin_memcpy(r[q].v, x + 16 * q * p.ldx, sizeof(r[q].v));
    } else {
#pragma unroll
        for (int q = 0; q < 8; ++q) {
            const bool in = q < rows;
            r[q] = raw8(x + (in ? 16 * q * p.ldx : 0), in ? cols : 0);
        }
    }
    float amax = 0.f;
#pragma unroll
    for (int q = 0; q < 8; ++q)
#pragma unroll
        for (int i = 0; i < 8; ++i) amax = fmaxf(amax, finite_abs(r[q].at(i)));
    amax = lanes_max<64>(amax);
    if ((threadIdx.x & 63) == 0) scratch[threadIdx.x >> 6] = amax;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kThreads / 64; ++i) amax = fmaxf(amax, scratch[i]);
    const float s = fp8_scale(amax);
#pragma unroll
    for (int q = 0; q < 8; ++q) {
        float v[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = r[q].at(i);
        if (whole || q < rows) store_fp8(q8 + 16 * q * p.ldq, whole ? 8 : cols, to_fp8(v, s));
    }
    if (threadIdx.x == 0) p.S[mb * p.lds + b] = s;
}

unsigned grid_of(int64_t groups) { return (unsigned)(groups < 1 << 20 ? groups : 1 << 20); }

// Calls f(threads, groups) with the threads that share a row of D columns and
// the groups of eight that each holds, as constants: a wave for short rows, the
// workgroup's four, sixteen.  False: more columns than registers hold.
template <int NT, int NV, typename F>
bool with_team_of(F &&f) {
    f(std::integral_constant<int, NT>(), std::integral_constant<int, NV>());
    return true;
}
template <typename F>
bool with_team(int64_t D, F &&f) {
    return D <= 512     ? with_team_of<64, 1>(f)
           : D <= 1024  ? with_team_of<64, 2>(f)
           : D <= 2048  ? with_team_of<64, 4>(f)
           : D <= 4096  ? with_team_of<256, 2>(f)
           : D <= 8192  ? with_team_of<256, 4>(f)
           : D <= 16384 ? with_team_of<1024, 2>(f)
                        : false;
}
// The gradient's, which holds three rows, the weight and its gradient's sums.
template <typename F>
bool with_backward_team(int64_t D, F &&f) {
    return D <= 512    ? with_team_of<64, 1>(f)
           : D <= 1024 ? with_team_of<64, 2>(f)
           : D <= 2048 ? with_team_of<256, 1>(f)
           : D <= 4096 ? with_team_of<256, 2>(f)
           : D <= 8192 ? with_team_of<1024, 1>(f)
                       : false;
}

}  // namespace

// Workgroups of the gradient's kernel: as many as its registers let the CUs hold,
// up to four each (8191x2048 with two 44.5 us, the rows in flight too few).
int norm_backward_slabs(int64_t T, int64_t D) {
    int64_t groups = T, most = 512;
    with_backward_team(D, [&](auto nt, auto nv) {
        groups = (T + RowTeam<nt()>::ROWS - 1) / RowTeam<nt()>::ROWS;
        most = nt() == 1024 ? 256 : nv() > 1 ? 768 : 1024;
    });
    return (int)(groups < most ? groups : most);
}

xtc_status launch_rmsnorm(const NormArgs &a, xtc_dtype dtype, bool quantize, hipStream_t s) {
    const bool done = with_team(a.D, [&](auto nt, auto nv) {
        constexpr int NT = nt(), NV = nv();
        const auto kernel = dtype == XTC_F32 ? (quantize ? rmsnorm_kernel<float, true, NT, NV> : rmsnorm_kernel<float, false, NT, NV>)
                                             : (quantize ? rmsnorm_kernel<Bf16, true, NT, NV> : rmsnorm_kernel<Bf16, false, NT, NV>);
        constexpr int ROWS = RowTeam<NT>::ROWS;
        const int64_t groups = (a.T + ROWS - 1) / ROWS;
        // (a launch has fewer than 2^32 threads)
        for (int64_t g = 0; g < groups; g += 1 << 21) {
            NormArgs b = a;
            const int64_t e = dtype == XTC_F32 ? 4 : 2, t0 = g * ROWS;
            auto on = [](const void *p, int64_t bytes) { return p ? (void *)(static_cast<char *>(const_cast<void *>(p)) + bytes) : nullptr; };
            b.T = a.T - t0 < (int64_t)ROWS << 21 ? a.T - t0 : (int64_t)ROWS << 21;
            b.X = on(a.X, t0 * a.ldx * e);
            b.R = on(a.R, t0 * a.ldr * e);
            b.Y = on(a.Y, t0 * a.ldy * (quantize ? 1 : e));
            b.S = static_cast<float *>(on(a.S, t0 * a.lds * 4));
            b.H = on(a.H, t0 * a.ldh * e);
            b.rstd = static_cast<float *>(on(a.rstd, t0 * 4));
            kernel<<<(unsigned)((b.T + ROWS - 1) / ROWS), RowTeam<NT>::THREADS, 0, s>>>(b);
        }
    });
    if (!done) {
        const auto kernel = dtype == XTC_F32 ? (quantize ? rmsnorm_loop_kernel<float, true> : rmsnorm_loop_kernel<float, false>)
                                             : (quantize ? rmsnorm_loop_kernel<Bf16, true> : rmsnorm_loop_kernel<Bf16, false>);
        kernel<<<grid_of(a.T), kThreads, 0, s>>>(a);
    }
    return hip_status(hipGetLastError());
}

xtc_status launch_rmsnorm_backward(const NormBackwardArgs &a, xtc_dtype dtype, hipStream_t s) {
    const int slabs = norm_backward_slabs(a.T, a.D);
    if (a.T > 0) {
        const bool done = with_backward_team(a.D, [&](auto nt, auto nv) {
            constexpr int NT = nt(), NV = nv();
            const auto kernel = dtype == XTC_F32 ? rmsnorm_backward_kernel<float, NT, NV> : rmsnorm_backward_kernel<Bf16, NT, NV>;
            kernel<<<(unsigned)slabs, RowTeam<NT>::THREADS, 0, s>>>(a);
        });
        if (!done) {
            const auto dx = dtype == XTC_F32 ? rmsnorm_dx_kernel<float> : rmsnorm_dx_kernel<Bf16>;
            const auto dw = dtype == XTC_F32 ? rmsnorm_dw_kernel<float> : rmsnorm_dw_kernel<Bf16>;
            dx<<<grid_of(a.T), kThreads, 0, s>>>(a);
            dw<<<dim3((unsigned)(((int64_t)a.D + kStep - 1) / kStep), (unsigned)slabs), kThreads, 0, s>>>(a);
        }
    }
    rmsnorm_dw_join_kernel<<<(unsigned)(((int64_t)a.D + kJoinColumns - 1) / kJoinColumns), kJoinThreads, 0, s>>>(a.partial, slabs, a.D, a.DW);
    return hip_status(hipGetLastError());
}

xtc_status launch_quantize(const QuantArgs &a, xtc_dtype dtype, hipStream_t s) {
    const int64_t kb = (a.K + kScaleBlock - 1) / kScaleBlock;
    if (a.block_rows == 1) {
        const auto kernel = dtype == XTC_F32 ? quantize_rows_kernel<float> : quantize_rows_kernel<Bf16>;
        kernel<<<grid_of((a.M * kb + 15) / 16), kThreads, 0, s>>>(a);
    } else {
        const int64_t blocks = (a.M + 127) / 128 * kb;
        if (blocks >= kMostGroups) return XTC_ERR_TOO_LARGE;
        const auto kernel = dtype == XTC_F32 ? quantize_blocks_kernel<float> : quantize_blocks_kernel<Bf16>;
        kernel<<<(unsigned)blocks, kThreads, 0, s>>>(a);
    }
    return hip_status(hipGetLastError());
}

}  // namespace xtc

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
                store_fp8(static_cast<uint8_t *>(p.Y) + t * p.ldy + c, valid, to_fp8(y, 1.f / s));
                if ((tid & 15) == 0 && valid > 0) p.S[t * p.lds + c / kScaleBlock] = s;
            } else {
                store8(static_cast<T *>(p.Y) + t * p.ldy + c, valid, y);
            }
        }
    }
}

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

// Column sums of the slabs, in their order.
__global__ void __launch_bounds__(kThreads) rmsnorm_dw_join_kernel(const float *partial, int slabs, int D, float *DW) {
    const int c = blockIdx.x * kThreads + threadIdx.x;
    if (c >= D) return;
    float sum = 0.f;
    for (int g = 0; g < slabs; ++g) sum += partial[(int64_t)g * D + c];
    DW[c] = sum;
}

// e4m3 with a scale per 1 x 128 block: sixteen lanes a block.
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
        store_fp8(p.Q + m * p.ldq + k, valid, to_fp8(v, 1.f / s));
        if (sub == 0) p.S[m * p.lds + (b - m * kb)] = s;
    }
}

// e4m3 with a scale per 128 x 128 block: a workgroup a block, which stays in
// registers between its maximum and its rounding.
template <typename T>
__global__ void __launch_bounds__(kThreads) quantize_blocks_kernel(QuantArgs p) {
    __shared__ float scratch[kThreads / 64];
    const int64_t kb = (p.K + kScaleBlock - 1) / kScaleBlock, blocks = (p.M + 127) / 128 * kb;
    const int sub = threadIdx.x & 15, row = threadIdx.x >> 4;
    for (int64_t b = blockIdx.x; b < blocks; b += gridDim.x) {
        const int64_t mb = b / kb, k = (b - mb * kb) * kScaleBlock + sub * 8, m = mb * 128 + row;
        const int cols = (int)(p.K - k < 8 ? p.K - k : 8);
        float v[8][8], amax = 0.f;
#pragma unroll
        for (int q = 0; q < 8; ++q) {
            const bool in = m + 16 * q < p.M;
            load8(static_cast<const T *>(p.X) + (in ? (m + 16 * q) * p.ldx + k : 0), in ? cols : 0, v[q]);
#pragma unroll
            for (int i = 0; i < 8; ++i) amax = fmaxf(amax, finite_abs(v[q][i]));
        }
        amax = lanes_max<64>(amax);
        __syncthreads();
        if ((threadIdx.x & 63) == 0) scratch[threadIdx.x >> 6] = amax;
        __syncthreads();
#pragma unroll
        for (int i = 0; i < kThreads / 64; ++i) amax = fmaxf(amax, scratch[i]);
        const float s = fp8_scale(amax), inv = 1.f / s;
#pragma unroll
        for (int q = 0; q < 8; ++q)
            if (m + 16 * q < p.M) store_fp8(p.Q + (m + 16 * q) * p.ldq + k, cols, to_fp8(v[q], inv));
        if (threadIdx.x == 0) p.S[mb * p.lds + (b - mb * kb)] = s;
    }
}

unsigned grid_of(int64_t groups) { return (unsigned)(groups < 1 << 20 ? groups : 1 << 20); }

}  // namespace

int norm_backward_slabs(int64_t T, int64_t) { return (int)(T < 256 ? T : 256); }

xtc_status launch_rmsnorm(const NormArgs &a, xtc_dtype dtype, bool quantize, hipStream_t s) {
    const auto kernel = dtype == XTC_F32 ? (quantize ? rmsnorm_loop_kernel<float, true> : rmsnorm_loop_kernel<float, false>)
                                         : (quantize ? rmsnorm_loop_kernel<Bf16, true> : rmsnorm_loop_kernel<Bf16, false>);
    kernel<<<grid_of(a.T), kThreads, 0, s>>>(a);
    return hip_status(hipGetLastError());
}

xtc_status launch_rmsnorm_backward(const NormBackwardArgs &a, xtc_dtype dtype, hipStream_t s) {
    const unsigned slabs = (unsigned)norm_backward_slabs(a.T, a.D);
    const unsigned wide = (unsigned)(((int64_t)a.D + kStep - 1) / kStep);
    if (a.T > 0) {
        const auto dx = dtype == XTC_F32 ? rmsnorm_dx_kernel<float> : rmsnorm_dx_kernel<Bf16>;
        const auto dw = dtype == XTC_F32 ? rmsnorm_dw_kernel<float> : rmsnorm_dw_kernel<Bf16>;
        dx<<<grid_of(a.T), kThreads, 0, s>>>(a);
        dw<<<dim3(wide, slabs), kThreads, 0, s>>>(a);
    }
    rmsnorm_dw_join_kernel<<<(a.D + kThreads - 1) / kThreads, kThreads, 0, s>>>(a.partial, (int)slabs, a.D, a.DW);
    return hip_status(hipGetLastError());
}

xtc_status launch_quantize(const QuantArgs &a, xtc_dtype dtype, hipStream_t s) {
    const int64_t kb = (a.K + kScaleBlock - 1) / kScaleBlock;
    if (a.block_rows == 1) {
        const auto kernel = dtype == XTC_F32 ? quantize_rows_kernel<float> : quantize_rows_kernel<Bf16>;
        kernel<<<grid_of((a.M * kb + 15) / 16), kThreads, 0, s>>>(a);
    } else {
        const auto kernel = dtype == XTC_F32 ? quantize_blocks_kernel<float> : quantize_blocks_kernel<Bf16>;
        kernel<<<grid_of((a.M + 127) / 128 * kb), kThreads, 0, s>>>(a);
    }
    return hip_status(hipGetLastError());
}

}  // namespace xtc

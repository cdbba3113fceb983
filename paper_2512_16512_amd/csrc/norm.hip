// Root-mean-square norm and layer norm (CENTER) with the residual's addition, their
// gradients, and the conversion of rows and blocks to e4m3 with a scale.
//
//   h = x + r, rstd = 1 / sqrt(mean_j h_j^2 + eps), y_j = w_j h_j rstd
//   centred: d = h - mean_j h_j, rstd = 1 / sqrt(mean_j d_j^2 + eps), y_j = w_j d_j rstd + b_j
//
// with h and every sum in fp32.  In 8 bits the 128 values of a block share
// s = max(amax / 448, 2^-126) and are rounded from y / s.
//
// The gradient, with xh = h rstd (centred: d rstd) and g = dy w:
//   dx = rstd (g - xh mean_j(g_j xh_j)) + dr,   dw_j = sum_t dy_tj xh_tj
//   centred: dx = rstd (g - mean_j g_j - xh mean_j(g_j xh_j)) + dr,   db_j = sum_t dy_tj
//
// The centred sum of squares is taken from the differences, in a second pass over
// registers: mean(h^2) - mean(h)^2 loses what a large mean leaves of 24 bits.
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
// The layer norm (CENTER) reads and writes past the caches: 8192 x 4096 bf16 with a residual 49 us, 5.5 TB/s of its
// 269 MB, as fast as a copy (64 through the caches; 103 with a wave a row, whose registers leave too few rows in
// flight; rows at odd addresses, 8192 x 3001, 52 and 60).
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

template <typename T, bool QUANT, bool CENTER, int NT, int NV>
__global__ void __launch_bounds__(RowTeam<NT>::THREADS) norm_kernel(NormArgs p) {
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
        rx[v] = CENTER ? raw8_once(x + c, D - c) : raw8(x + c, D - c);
        if (r) rr[v] = CENTER ? raw8_once(r + c, D - c) : raw8(r + c, D - c);
    }
    float h[NV][8], sum = 0.f;
#pragma unroll
    for (int v = 0; v < NV; ++v)
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            h[v][i] = r ? rx[v].at(i) + rr[v].at(i) : rx[v].at(i);
            sum += CENTER ? h[v][i] : h[v][i] * h[v][i];
        }
    sum = Team::sum(sum, scratch);
    float mean = 0.f;
    if constexpr (CENTER) {
        mean = sum / (float)D;
        sum = 0.f;
#pragma unroll
        for (int v = 0; v < NV; ++v)
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float d = (v * NT + tid) * 8 + i < D ? h[v][i] - mean : 0.f;
                sum += d * d;
            }
        sum = Team::sum(sum, scratch);
        if (tid == 0 && p.mean) p.mean[t] = mean;
    }
    const float rstd = 1.f / sqrtf(sum / (float)D + p.eps);
    if (tid == 0 && p.rstd) p.rstd[t] = rstd;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
        const int c = (v * NT + tid) * 8, valid = D - c;
        const Raw8<float> w = raw_weight(p.W, p.w_f32, x, c, valid);
        if (p.H) (CENTER ? store8_past<T> : store8<T>)(static_cast<T *>(p.H) + t * p.ldh + c, valid, h[v]);
        Raw8<float> b = {};
        if constexpr (CENTER) {
            if (p.B) b = raw_weight(p.B, p.w_f32, x, c, valid);
        }
        float y[8], amax = 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            y[i] = CENTER ? (h[v][i] - mean) * rstd * w.v[i] + b.v[i] : h[v][i] * rstd * w.v[i];
            // (columns past the end, which would be b - mean rstd w, are zeros already: w and b are)
            if constexpr (QUANT) amax = fmaxf(amax, finite_abs(y[i]));
        }
        if constexpr (QUANT) {
            const float s = fp8_scale(lanes_max<16>(amax));
            store_fp8(static_cast<uint8_t *>(p.Y) + t * p.ldy + c, valid, to_fp8(y, s));
            if ((tid & 15) == 0 && valid > 0) p.S[t * p.lds + c / kScaleBlock] = s;
        } else {
            (CENTER ? store8_past<T> : store8<T>)(static_cast<T *>(p.Y) + t * p.ldy + c, valid, y);
        }
    }
}

// A workgroup per row, any number of columns: a pass for the sum of squares
// (CENTER: one for the mean before it), another that reads the row again.
template <typename T, bool QUANT, bool CENTER>
__global__ void __launch_bounds__(kThreads) norm_loop_kernel(NormArgs p) {
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
        float sum = 0.f, mean = 0.f;
        if constexpr (CENTER) {
            for (int c = tid * 8; c < D; c += kStep) {
                float h[8];
                load_h(c, h);
#pragma unroll
                for (int i = 0; i < 8; ++i) sum += h[i];
            }
            mean = group_sum(sum, scratch) / (float)D;
            if (tid == 0 && p.mean) p.mean[t] = mean;
            sum = 0.f;
        }
        for (int c = tid * 8; c < D; c += kStep) {
            float h[8];
            load_h(c, h);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float d = CENTER ? (c + i < D ? h[i] - mean : 0.f) : h[i];
                sum += d * d;
            }
        }
        sum = group_sum(sum, scratch);
        const float rstd = 1.f / sqrtf(sum / (float)D + p.eps);
        if (tid == 0 && p.rstd) p.rstd[t] = rstd;
        // (whole trips: the lanes that share a block's scale stay together)
        for (int c0 = 0; c0 < D; c0 += kStep) {
            const int c = c0 + tid * 8, valid = D - c;
            float h[8], w[8], b[8] = {}, y[8];
            load_h(c, h);
            load_weight(p.W, p.w_f32, x, c, valid, w);
            if constexpr (CENTER) {
                if (p.B) load_weight(p.B, p.w_f32, x, c, valid, b);
            }
            if (p.H) store8(static_cast<T *>(p.H) + t * p.ldh + c, valid, h);
#pragma unroll
            for (int i = 0; i < 8; ++i) y[i] = CENTER ? (h[i] - mean) * rstd * w[i] + b[i] : h[i] * rstd * w[i];
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
// the sums over its rows of its columns' part of DW (CENTER: and of DB), and the
// workgroup leaves one row of partial sums (CENTER: of 2D, DW's first; TEAMS of NT threads share it, so that
// there are 256 such rows at most, and both sums of a row pass one barrier).  The next row is on its way while one is computed.
// 8191 x 2048 bf16, bound by memory: 28.6 us, 4.7 TB/s; DX and DW by kernels of
// their own, which read the rows twice, took 151 us.  The layer norm's, past the caches: 28.6 us and 4 for the join of
// 256 rows of 4096 sums (37 us in all through the caches with 1024 rows of sums and two barriers a row, so 31).
template <typename T, bool CENTER, int NT, int NV, int TEAMS>
__global__ void __launch_bounds__(NT * TEAMS) norm_backward_kernel(NormBackwardArgs p) {
    typedef RowTeam<NT> Team;
    __shared__ float scratch[NT / 64];
    __shared__ float two[CENTER ? 2 : 1][TEAMS][NT / 64][2];          // the centred sums, of two trips in turn
    __shared__ float sums[TEAMS > 1 ? (TEAMS - 1) * NT * NV * 8 : 1];   // of the workgroup's other teams
    constexpr int NB = CENTER ? NV : 1;
    const int tid = threadIdx.x % NT, team = threadIdx.x / NT, D = p.D;
    const int64_t step = (int64_t)gridDim.x * TEAMS;
    Raw8<T> rx[NV], ry[NV], rr[NV];
    float w[NV][8], dw[NV][8], db[NB][8], rstd_next = 0.f, mean_next = 0.f;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
        const int c = (v * NT + tid) * 8;
        const Raw8<float> q = raw_weight(p.W, p.w_f32, static_cast<const T *>(nullptr), c, D - c);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            w[v][i] = q.v[i];
            dw[v][i] = 0.f;
            if constexpr (CENTER) db[v][i] = 0.f;
        }
    }
    auto fetch = [&](int64_t t) {
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            const int c = (v * NT + tid) * 8, valid = t < p.T ? D - c : 0;
            const auto read = CENTER ? raw8_once<T> : raw8<T>;
            rx[v] = read(static_cast<const T *>(p.X) + t * p.ldx + c, valid);
            ry[v] = read(static_cast<const T *>(p.DY) + t * p.lddy + c, valid);
            if (p.DR) rr[v] = read(static_cast<const T *>(p.DR) + t * p.lddr + c, valid);
        }
        rstd_next = t < p.T ? p.rstd[t] : 0.f;
        if constexpr (CENTER) mean_next = t < p.T ? p.mean[t] : 0.f;
    };
    // (every team of a workgroup takes part in every trip: the sums below have barriers)
    int64_t t = (int64_t)blockIdx.x * TEAMS + team;
    int turn = 0;
    fetch(t);
    for (int64_t t0 = (int64_t)blockIdx.x * TEAMS; t0 < p.T; t0 += step, t += step) {
        const float rstd = rstd_next, centre = mean_next;
        float h[NV][8], g[NV][8], d[NV][8], sum = 0.f, sum_g = 0.f;
#pragma unroll
        for (int v = 0; v < NV; ++v)
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                // (past the end y and w are zeros; -centre * rstd, which may leave fp32, is none)
                h[v][i] = !CENTER                          ? rx[v].at(i) * rstd
                          : (v * NT + tid) * 8 + i < D ? (rx[v].at(i) - centre) * rstd
                                                       : 0.f;
                const float y = ry[v].at(i);
                dw[v][i] += y * h[v][i];
                if constexpr (CENTER) db[v][i] += y;
                g[v][i] = y * w[v][i];
                if constexpr (CENTER) sum_g += g[v][i];
                d[v][i] = p.DR ? rr[v].at(i) : 0.f;
                sum += g[v][i] * h[v][i];
            }
        fetch(t + step);
        float mean_g = 0.f;
        if constexpr (CENTER) {
            // both sums at once; what a wave still reads of one trip the next does not write
            sum = lanes_sum<64>(sum);
            sum_g = lanes_sum<64>(sum_g);
            if constexpr (NT > 64) {
                float (&at)[NT / 64][2] = two[turn][team];
                if ((tid & 63) == 0) {
                    at[tid >> 6][0] = sum;
                    at[tid >> 6][1] = sum_g;
                }
                __syncthreads();
                sum = sum_g = 0.f;
#pragma unroll
                for (int i = 0; i < NT / 64; ++i) {
                    sum += at[i][0];
                    sum_g += at[i][1];
                }
                turn ^= 1;
            }
            mean_g = sum_g / (float)D;
        } else {
            sum = Team::sum(sum, scratch);
        }
        const float mean = sum / (float)D;
        if (t < p.T) {
#pragma unroll
            for (int v = 0; v < NV; ++v) {
                const int c = (v * NT + tid) * 8;
                float o[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) o[i] = d[v][i] + rstd * (CENTER ? g[v][i] - mean_g - h[v][i] * mean : g[v][i] - h[v][i] * mean);
                store8_to(static_cast<T *>(p.DX) + t * p.lddx + c, D - c, o, CENTER && p.past);
            }
        }
    }
    // the other teams' sums are added, and the workgroup's row of them written
    auto leave = [&](auto &sum, float *to) __attribute__((always_inline)) {
        if constexpr (TEAMS > 1) {
            if (team > 0) {
#pragma unroll
                for (int v = 0; v < NV; ++v)
#pragma unroll
                    for (int i = 0; i < 8; ++i) sums[((team - 1) * NV * 8 + v * 8 + i) * NT + tid] = sum[v][i];
            }
            __syncthreads();
            if (team == 0) {
#pragma unroll
                for (int v = 0; v < NV; ++v)
#pragma unroll
                    for (int i = 0; i < 8; ++i)
#pragma unroll
                        for (int q = 0; q < TEAMS - 1; ++q) sum[v][i] += sums[(q * NV * 8 + v * 8 + i) * NT + tid];
            }
        }
        if (team == 0) {
#pragma unroll
            for (int v = 0; v < NV; ++v) {
                const int c = (v * NT + tid) * 8;
                store8(to + c, D - c, sum[v]);
            }
        }
    };
    float *to = p.partial + (int64_t)blockIdx.x * D * (CENTER ? 2 : 1);
    leave(dw, to);
    if constexpr (CENTER) {
        __syncthreads();
        leave(db, to + D);
    }
}

// Rows of more columns than registers hold: DX and DW by kernels of their own, which
// read X and DY three times in all (4096 x 16384 bf16: 311 us, 1.7 TB/s of what one
// pass would move; 4096 x 8192 in one pass 64 us, 4.2 TB/s, the layer norm's too).
template <typename T>
__global__ void __launch_bounds__(kThreads) norm_dx_kernel(NormBackwardArgs p) {
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

// A row of the layer norm's DX, held in registers between its sums and its outputs, NV groups of eight columns a thread; wider
// rows (NV 0) are read twice.
template <typename T, int NT, int NV>
__device__ __forceinline__ void layernorm_dx_rows(const NormBackwardArgs &p, int64_t first, int64_t step, float (&both)[2][NT / 64]) {
    constexpr int HELD = NV > 0 ? NV : 1;
    const int tid = threadIdx.x, D = p.D;
    for (int64_t t = first; t < p.T; t += step) {
        const T *x = static_cast<const T *>(p.X) + t * p.ldx;
        const T *dy = static_cast<const T *>(p.DY) + t * p.lddy;
        const float rstd = p.rstd[t], centre = p.mean[t];
        Raw8<T> rx[HELD], ry[HELD];
        float sum = 0.f, sum_g = 0.f;
        auto add = [&](int c, const Raw8<T> &a, const Raw8<T> &b) __attribute__((always_inline)) {
            const Raw8<float> w = raw_weight(p.W, p.w_f32, x, c, D - c);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                // (past the end b and w are zeros; -centre * rstd, which may leave fp32, is none)
                const float g = b.at(i) * w.v[i];
                sum += g * (c + i < D ? (a.at(i) - centre) * rstd : 0.f);
                sum_g += g;
            }
        };
        if constexpr (NV > 0) {
#pragma unroll
            for (int v = 0; v < NV; ++v) {
                const int c = (v * NT + tid) * 8;
                rx[v] = raw8(x + c, D - c);
                ry[v] = raw8(dy + c, D - c);
            }
#pragma unroll
            for (int v = 0; v < NV; ++v) add((v * NT + tid) * 8, rx[v], ry[v]);
        } else {
            for (int c = tid * 8; c < D; c += NT * 8) add(c, raw8(x + c, D - c), raw8(dy + c, D - c));
        }
        sum = lanes_sum<64>(sum);
        sum_g = lanes_sum<64>(sum_g);
        __syncthreads();
        if ((tid & 63) == 0) {
            both[0][tid >> 6] = sum;
            both[1][tid >> 6] = sum_g;
        }
        __syncthreads();
        sum = sum_g = 0.f;
#pragma unroll
        for (int i = 0; i < NT / 64; ++i) {
            sum += both[0][i];
            sum_g += both[1][i];
        }
        const float mean = sum / (float)D, mean_g = sum_g / (float)D;
        auto write = [&](int c, const Raw8<T> &a, const Raw8<T> &b) __attribute__((always_inline)) {
            const Raw8<float> w = raw_weight(p.W, p.w_f32, x, c, D - c);
            Raw8<T> r = {};
            if (p.DR) r = raw8(static_cast<const T *>(p.DR) + t * p.lddr + c, D - c);
            float o[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) o[i] = r.at(i) + rstd * (b.at(i) * w.v[i] - mean_g - (a.at(i) - centre) * rstd * mean);
            store8_to(static_cast<T *>(p.DX) + t * p.lddx + c, D - c, o, p.past);
        };
        if constexpr (NV > 0) {
#pragma unroll
            for (int v = 0; v < NV; ++v) write((v * NT + tid) * 8, rx[v], ry[v]);
        } else {
            for (int c = tid * 8; c < D; c += NT * 8) write(c, raw8(x + c, D - c), raw8(dy + c, D - c));
        }
    }
}

// The layer norm's DW and DB take the rows' mean and rstd, but no sums of theirs: workgroups of 64 columns and a slab of rows
// (eight lanes of eight columns, NT / 8 rows at once) leave them beside those of the rows.  X and DY are read twice (rows of
// more than 16384 columns three times), but few rows take one launch, and no thread holds columns' sums over its rows.  64 x
// 1152 bf16 4.4 us (in two launches 9.7); 4096 x 16384 227 us, 2.4 TB/s of what one pass would move (DX and DW one after the
// other 330; one pass spills 160 registers of 1024 threads, 300 of 512).
constexpr int kFewColumns = 64, kFewLanes = kFewColumns / 8;
template <typename T, int NT, int NV>
__global__ void __launch_bounds__(NT) norm_apart_backward_kernel(NormBackwardArgs p, int column_groups, int slabs) {
    constexpr int TEAMS = NT / kFewLanes;
    __shared__ __attribute__((aligned(16))) float sums[2][TEAMS][kFewColumns];
    const int before = column_groups * slabs, id = (int)blockIdx.x;
    if (id >= before) {
        __shared__ float both[2][NT / 64];
        layernorm_dx_rows<T, NT, NV>(p, id - before, (int)gridDim.x - before, both);
        return;
    }
    const int lane = threadIdx.x % kFewLanes, team = threadIdx.x / kFewLanes, slab = id / column_groups;
    const int64_t step = (int64_t)slabs * TEAMS;
    for (int c0 = (id - slab * column_groups) * kFewColumns; c0 < p.D; c0 += column_groups * kFewColumns) {
        const int c = c0 + lane * 8, valid = p.D - c;
        float sum[2][8] = {};
        constexpr int AT_ONCE = 4;
        for (int64_t t = (int64_t)slab * TEAMS + team; t < p.T; t += AT_ONCE * step) {
            Raw8<T> x[AT_ONCE], y[AT_ONCE];
            float rstd[AT_ONCE], centre[AT_ONCE];
#pragma unroll
            for (int r = 0; r < AT_ONCE; ++r) {
                // (past the last row that one again: loads in a branch would wait for it)
                const int64_t at = t + r * step < p.T ? t + r * step : p.T - 1;
                x[r] = raw8(static_cast<const T *>(p.X) + at * p.ldx + c, valid);
                y[r] = raw8(static_cast<const T *>(p.DY) + at * p.lddy + c, valid);
                rstd[r] = p.rstd[at];
                centre[r] = p.mean[at];
            }
#pragma unroll
            for (int r = 0; r < AT_ONCE; ++r)
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const bool in = t + r * step < p.T;
                    sum[0][i] += in ? y[r].at(i) * ((x[r].at(i) - centre[r]) * rstd[r]) : 0.f;
                    sum[1][i] += in ? y[r].at(i) : 0.f;
                }
        }
#pragma unroll
        for (int k = 0; k < 2; ++k) __builtin_memcpy(__builtin_assume_aligned(&sums[k][team][lane * 8], 16), sum[k], sizeof(sum[k]));
        __syncthreads();
        if (threadIdx.x < 2 * kFewColumns) {
            const int k = threadIdx.x / kFewColumns, q = threadIdx.x % kFewColumns, at = c0 + q;
            float s = 0.f;
#pragma unroll
            for (int i = 0; i < TEAMS; ++i) s += sums[k][i][q];
            if (at < p.D) (slabs > 1 ? p.partial + ((int64_t)slab * 2 + k) * p.D : k ? p.DB : p.DW)[at] = s;
        }
        __syncthreads();
    }
}

// Sums of dy * xh over the slab blockIdx.y of rows.
template <typename T>
__global__ void __launch_bounds__(kThreads) norm_dw_kernel(NormBackwardArgs p) {
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
__global__ void __launch_bounds__(kJoinThreads) column_sums_kernel(const float *partial, int slabs, int D, float *DW, float *DB, int64_t first) {
    __shared__ float s[kJoinThreads];
    const int run = threadIdx.x / kJoinColumns;
    // (with DB: 2D sums a slab)
    const int64_t c = first + (int64_t)blockIdx.x * kJoinColumns + threadIdx.x % kJoinColumns, columns = DB ? 2 * (int64_t)D : D;
    constexpr int RUNS = kJoinThreads / kJoinColumns;
    float sum = 0.f;
    if (c < columns) {
#pragma unroll 8
        for (int g = run; g < slabs; g += RUNS) sum += partial[g * columns + c];
    }
    s[threadIdx.x] = sum;
#pragma unroll
    for (int half = RUNS / 2; half > 0; half /= 2) {
        __syncthreads();
        if (run < half) s[threadIdx.x] += s[threadIdx.x + half * kJoinColumns];
    }
    if (run == 0 && c < columns) (c < D ? DW : DB - D)[c] = s[threadIdx.x];
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

// Whether the layer norm's gradient goes by norm_apart_backward_kernel, and its slabs of rows there: one and a single launch
// up to kFewRows, and many rows of what registers hold with their sums as long as the caches have them when they are read
// again (bf16, us, apart and not: 1024 x 4096 14.5 and 20.1, 2048 x 4096 20.5 and 25.3, 4096 x 4096 36.7 and 35.8; 1024 x 600
// 11.3 and 9.6).
constexpr int kFewRows = 256, kApartSlabs = 64;
bool apart(int64_t T, int64_t D) { return D > 8192 || T <= kFewRows || (D > 1024 && T <= 2048); }
int apart_slabs(int64_t T) { return (int)(T <= kFewRows ? 1 : T <= kFewRows * kApartSlabs ? (T + kFewRows - 1) / kFewRows : kApartSlabs); }

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
// The gradient's, which holds three rows, the weight and its gradient's sums: f(threads, groups, teams of a
// workgroup).
template <int NT, int NV, int TEAMS, typename F>
bool with_teams_of(F &&f) {
    f(std::integral_constant<int, NT>(), std::integral_constant<int, NV>(), std::integral_constant<int, TEAMS>());
    return true;
}
template <bool CENTER, typename F>
bool with_backward_team(int64_t D, F &&f) {
    constexpr bool C = CENTER;
    return D <= 512    ? with_teams_of<64, 1, C ? 16 : 4>(f)
           : D <= 1024 ? with_teams_of<C ? 128 : 64, C ? 1 : 2, C ? 8 : 4>(f)
           : D <= 2048 ? with_teams_of<256, 1, C ? 4 : 1>(f)
           : D <= 4096 ? with_teams_of<C ? 512 : 256, C ? 1 : 2, C ? 2 : 1>(f)
           : D <= 8192 ? with_teams_of<1024, 1, 1>(f)
                       : false;
}

}  // namespace

// Workgroups of the gradient's kernel: as many as its registers let the CUs hold,
// up to four each (8191x2048 with two 44.5 us, the rows in flight too few).
// (CENTER, of two sums a column: teams share a workgroup, whose sums are one row.)
template <bool CENTER>
static int backward_slabs(int64_t T, int64_t D) {
    if (CENTER && apart(T, D)) return T > 0 ? apart_slabs(T) : 0;
    int64_t groups = T, most = 512;
    with_backward_team<CENTER>(D, [&](auto nt, auto nv, auto teams) {
        groups = (T + teams() - 1) / teams();
        most = nt() == 1024 ? 256 : nv() > 1 ? 768 : 1024;
        if (CENTER) most = 256;
    });
    return (int)(groups < most ? groups : most);
}
int norm_backward_slabs(int64_t T, int64_t D) { return backward_slabs<false>(T, D); }
int layernorm_backward_slabs(int64_t T, int64_t D) { return backward_slabs<true>(T, D); }

xtc_status launch_column_sums(const float *partial, int slabs, int D, float *DW, float *DB, hipStream_t s) {
    const int64_t columns = DB ? 2 * (int64_t)D : D;
    // (a launch has fewer than 2^32 threads)
    constexpr int64_t kMost = (int64_t(1) << 31) / kJoinThreads * kJoinColumns;
    for (int64_t first = 0; first < columns; first += kMost) {
        const int64_t n = columns - first < kMost ? columns - first : kMost;
        column_sums_kernel<<<(unsigned)((n + kJoinColumns - 1) / kJoinColumns), kJoinThreads, 0, s>>>(partial, slabs, D, DW, DB, first);
    }
    return hip_status(hipGetLastError());
}

namespace {

template <bool CENTER>
xtc_status launch_norm(const NormArgs &a, xtc_dtype dtype, bool quantize, hipStream_t s) {
    auto run = [&](auto nt, auto nv) {
        constexpr int NT = nt(), NV = nv();
        const auto kernel = dtype == XTC_F32 ? (quantize ? norm_kernel<float, true, CENTER, NT, NV> : norm_kernel<float, false, CENTER, NT, NV>)
                                             : (quantize ? norm_kernel<Bf16, true, CENTER, NT, NV> : norm_kernel<Bf16, false, CENTER, NT, NV>);
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
            b.mean = static_cast<float *>(on(a.mean, t0 * 4));
            kernel<<<(unsigned)((b.T + ROWS - 1) / ROWS), RowTeam<NT>::THREADS, 0, s>>>(b);
        }
    };
    const bool done = with_team(a.D, run);
    if (!done) {
        const auto kernel = dtype == XTC_F32 ? (quantize ? norm_loop_kernel<float, true, CENTER> : norm_loop_kernel<float, false, CENTER>)
                                             : (quantize ? norm_loop_kernel<Bf16, true, CENTER> : norm_loop_kernel<Bf16, false, CENTER>);
        kernel<<<grid_of(a.T), kThreads, 0, s>>>(a);
    }
    return hip_status(hipGetLastError());
}

template <bool CENTER>
xtc_status launch_norm_backward(const NormBackwardArgs &a, xtc_dtype dtype, hipStream_t s) {
    const int slabs = backward_slabs<CENTER>(a.T, a.D);
    if (CENTER && a.T > 0 && apart(a.T, a.D)) {
        const int64_t across = ((int64_t)a.D + kFewColumns - 1) / kFewColumns, groups = across < 1 << 16 ? across : 1 << 16;
        const int64_t rows = a.T < 1 << 20 ? a.T : 1 << 20;
        auto run = [&](auto nt, auto nv) {
            const auto kernel = dtype == XTC_F32 ? norm_apart_backward_kernel<float, nt(), nv()> : norm_apart_backward_kernel<Bf16, nt(), nv()>;
            kernel<<<(unsigned)(groups * slabs + rows), nt(), 0, s>>>(a, (int)groups, slabs);
        };
        typedef std::integral_constant<int, kThreads> Threads;
        if (a.D <= kStep) run(Threads(), std::integral_constant<int, 1>());
        else if (a.D <= 2 * kStep) run(Threads(), std::integral_constant<int, 2>());
        else if (a.D <= 4 * kStep) run(Threads(), std::integral_constant<int, 4>());
        else if (a.D <= 8 * kStep) run(std::integral_constant<int, 2 * kThreads>(), std::integral_constant<int, 4>());
        else run(Threads(), std::integral_constant<int, 0>());
        const xtc_status st = hip_status(hipGetLastError());
        if (st != XTC_OK || slabs == 1) return st;
    } else if (a.T > 0) {
        const bool done = with_backward_team<CENTER>(a.D, [&](auto nt, auto nv, auto teams) {
            constexpr int NT = nt(), NV = nv(), TEAMS = teams();
            const auto kernel = dtype == XTC_F32 ? norm_backward_kernel<float, CENTER, NT, NV, TEAMS> : norm_backward_kernel<Bf16, CENTER, NT, NV, TEAMS>;
            kernel<<<(unsigned)slabs, NT * TEAMS, 0, s>>>(a);
        });
        if constexpr (!CENTER) if (!done) {
            const auto dx = dtype == XTC_F32 ? norm_dx_kernel<float> : norm_dx_kernel<Bf16>;
            const auto dw = dtype == XTC_F32 ? norm_dw_kernel<float> : norm_dw_kernel<Bf16>;
            dx<<<grid_of(a.T), kThreads, 0, s>>>(a);
            dw<<<dim3((unsigned)(((int64_t)a.D + kStep - 1) / kStep), (unsigned)slabs), kThreads, 0, s>>>(a);
        }
    }
    return launch_column_sums(a.partial, slabs, a.D, a.DW, CENTER ? a.DB : nullptr, s);
}

}  // namespace

xtc_status launch_rmsnorm(const NormArgs &a, xtc_dtype dtype, bool quantize, hipStream_t s) {
    return launch_norm<false>(a, dtype, quantize, s);
}
xtc_status launch_layernorm(const NormArgs &a, xtc_dtype dtype, bool quantize, hipStream_t s) {
    return launch_norm<true>(a, dtype, quantize, s);
}
xtc_status launch_rmsnorm_backward(const NormBackwardArgs &a, xtc_dtype dtype, hipStream_t s) {
    return launch_norm_backward<false>(a, dtype, s);
}
xtc_status launch_layernorm_backward(const NormBackwardArgs &given, xtc_dtype dtype, hipStream_t s) {
    NormBackwardArgs a = given;
    a.past = whole_lines(a.DX, a.lddx, dtype == XTC_F32 ? 4 : 2);
    return launch_norm_backward<true>(a, dtype, s);
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

// Internal interface between the host side of the 8-bit, grouped and
// normalisation operators (operators_api.cpp) and their kernels (norm.hip and
// grouped.hip, grouped_tile.hip, grouped_stream.hip).  Not installed.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/xtc.h"

namespace xtc {

// xtc_status of a HIP call; keeps the code of a failed one for xtc_last_hip_error.
xtc_status hip_status(hipError_t e);

constexpr int kScaleBlock = 128;   // consecutive values of a row that share a scale

// One launch over T rows of D columns.  Row strides are in elements.
struct NormArgs {
    int64_t T;
    int D;
    const void *X;
    int64_t ldx;
    const void *R;      // residual, added to X (null: none)
    int64_t ldr;
    const void *W;
    int w_f32;          // the weight is fp32 (else of X's type)
    float eps;
    void *Y;            // X's type, or e4m3 with scales S
    int64_t ldy;
    float *S;
    int64_t lds;
    void *H;            // X + R (null: not kept)
    int64_t ldh;
    float *rstd;        // null: not kept
};

struct NormBackwardArgs {
    int64_t T;
    int D;
    const void *DY;
    int64_t lddy;
    const void *X;
    int64_t ldx;
    const void *W;
    int w_f32;
    const float *rstd;
    const void *DR;     // gradient of the sum itself (null: none)
    int64_t lddr;
    void *DX;
    int64_t lddx;
    float *DW;
    float *partial;     // norm_backward_slabs(T) x D sums of a slab of rows each
};

struct QuantArgs {
    int64_t M, K;
    const void *X;
    int64_t ldx;
    int block_rows;     // 1 or 128
    uint8_t *Q;
    int64_t ldq;
    float *S;
    int64_t lds;
};

// A family of products C = A B with the rows of A in G consecutive groups,
// each with its own B (ends null: one group of all T rows).
struct GroupedArgs {
    int64_t T;          // rows of A
    int N, K;
    const void *A;
    int64_t lda;
    const float *SA;    // e4m3: a scale per row and 128 k, row stride ldsa
    int64_t ldsa;
    const void *B;      // of group g: B + g * stride_b elements
    int64_t ldb, stride_b;
    const float *SB;    // e4m3: a scale per 128 rows of B and 128 k
    int64_t ldsb, stride_sb;
    void *C;
    int64_t ldc;
    int64_t stride_c;   // the weights' gradient: C of group g at C + g * stride_c
    const int32_t *ends;
    int G;
    int out_bf16;       // C is bf16 (else fp32)
    int relu;
};

// Workgroups of a launch: fewer than 2^32 threads of 256 a workgroup.
constexpr int64_t kMostGroups = int64_t(1) << 24;

int norm_backward_slabs(int64_t T, int64_t D);
xtc_status launch_rmsnorm(const NormArgs &a, xtc_dtype dtype, bool quantize, hipStream_t s);
xtc_status launch_rmsnorm_backward(const NormBackwardArgs &a, xtc_dtype dtype, hipStream_t s);
xtc_status launch_quantize(const QuantArgs &a, xtc_dtype dtype, hipStream_t s);

// e4m3 A [T, K], B [N, K]
xtc_status launch_grouped_fp8(const GroupedArgs &a, hipStream_t s);
// bf16 A [T, K], B [K, N] (b_rows_n: [N, K])
xtc_status launch_grouped_bf16(const GroupedArgs &a, bool b_rows_n, hipStream_t s);
// bf16 A [T, K] and B [T, N]: C of group g [K, N] = A_g^T B_g
xtc_status launch_grouped_wgrad(const GroupedArgs &a, hipStream_t s);

// Which of the kernels for aligned rows a product takes (-1: the one for rows at
// any address), and how many there are.  kind: 0 e4m3, 1 bf16 with B [K, N], 2 with
// B [N, K], 3 a weights' gradient.
int grouped_kernel(const GroupedArgs &a, int kind, int *kernels);

}  // namespace xtc

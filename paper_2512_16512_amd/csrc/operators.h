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
    const void *B;      // layer norm: added last, of W's type (null: nothing)
    float *mean;        // layer norm (null: not kept)
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
    float *partial;     // norm_backward_slabs() x D (layer norm: layernorm_backward_slabs() x 2D) sums of a slab of rows each
    const float *mean;  // layer norm
    float *DB;
    int past;           // layer norm: DX's rows begin at 16 bytes
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

// A linear layer: one product of a family (ends null, G 1), and what follows it.
struct LinearArgs : GroupedArgs {
    const void *bias;   // N values (null: none)
    int bias_f32;       // else bf16; likewise the residual
    const void *R;      // T x N, added last (null: none)
    int64_t ldr;
    int r_f32;
    void *Z;            // what the activation takes, of C's type (null: not kept)
    int64_t ldz;
    int act;            // xtc_activation
    int splits;         // parts of the reduction, k_each long but the last
    int k_each;
    float *part;        // several splits: their sums, splits x rows x N
};

struct ActivationArgs {
    int64_t T;
    int N;
    const void *DY;
    int64_t lddy;
    int dy_f32;         // else bf16; likewise Z
    const void *Z;
    int64_t ldz;
    int z_f32;
    int act;
    void *DZ;           // bf16
    int64_t lddz;
    int past;           // DZ's rows begin at 16 bytes
    float *DB;          // column sums of the unrounded DZ (null: not wanted)
    float *partial;     // activation_slabs() x N sums of a slab of rows each
};

struct RouteArgs {
    int64_t T;
    int E, top;
    const void *scores;
    int64_t lds;
    const uint8_t *mask;    // 0: the token has no experts (null: every token has)
    int32_t *expert;        // T x top, like p and row
    float *p;
    int32_t *row;
    int32_t *token;         // T * top
    int32_t *counts, *ends; // E
    float *loss;
    int each;               // tokens of a workgroup
    int32_t *counts_of;     // of each workgroup: E counts and E sums, in whole fours
    float *sums_of;
};

struct RouteBackwardArgs {
    int64_t T;
    int E, top;
    const float *DP;        // null: zeros
    const void *scores;
    int64_t lds;
    const int32_t *expert;
    const float *p;
    const int32_t *counts;
    float dloss;
    void *DS;
    int64_t ldds;
};

struct CombineArgs {
    int64_t T, R;           // tokens; rows that there are
    int top, D;
    const void *rows;
    int64_t ldrows;
    const int32_t *row;     // T x top, like P
    const float *P;         // null: ones
    const void *RES;        // null: nothing added
    int64_t ldr;
    void *out;
    int64_t ldo;
};

struct CombineBackwardArgs {
    int64_t T, R;
    int top, D;
    const void *DOUT;
    int64_t lddo;
    const void *rows;
    int64_t ldrows;
    const int32_t *row, *token;
    const float *P;
    void *DROWS;
    int64_t lddr;
    int past;               // DROWS' rows begin at 16 bytes
    float *DP;
};

// Workgroups of a launch: fewer than 2^32 threads of 256 a workgroup.
constexpr int64_t kMostGroups = int64_t(1) << 24;

int norm_backward_slabs(int64_t T, int64_t D);
int layernorm_backward_slabs(int64_t T, int64_t D);
xtc_status launch_rmsnorm(const NormArgs &a, xtc_dtype dtype, bool quantize, hipStream_t s);
xtc_status launch_rmsnorm_backward(const NormBackwardArgs &a, xtc_dtype dtype, hipStream_t s);
xtc_status launch_layernorm(const NormArgs &a, xtc_dtype dtype, bool quantize, hipStream_t s);
xtc_status launch_layernorm_backward(const NormBackwardArgs &a, xtc_dtype dtype, hipStream_t s);
// DW = column sums of `slabs` rows of D values (with DB: of 2D, the second half its), in a fixed order.
xtc_status launch_column_sums(const float *partial, int slabs, int D, float *DW, float *DB, hipStream_t s);
xtc_status launch_quantize(const QuantArgs &a, xtc_dtype dtype, hipStream_t s);

// e4m3 A [T, K], B [N, K]
xtc_status launch_grouped_fp8(const GroupedArgs &a, hipStream_t s);
// bf16 A [T, K], B [K, N] (b_rows_n: [N, K])
xtc_status launch_grouped_bf16(const GroupedArgs &a, bool b_rows_n, hipStream_t s);
// bf16 A [T, K] and B [T, N]: C of group g [K, N] = A_g^T B_g
xtc_status launch_grouped_wgrad(const GroupedArgs &a, hipStream_t s);

// bf16 A [T, K] and B [K, N] (b_rows_n: [N, K]), with a workspace of linear_workspace() bytes (of fewer:
// XTC_ERR_BAD_SHAPE, before any HIP call).
int64_t linear_workspace(const LinearArgs &a, bool b_rows_n);
xtc_status launch_linear(const LinearArgs &a, bool b_rows_n, void *workspace, int64_t bytes, hipStream_t s);
// C [K, N] = A^T B of bf16 A [T, K], B [T, N]
int64_t linear_wgrad_workspace(const LinearArgs &a);
xtc_status launch_linear_wgrad(const LinearArgs &a, void *workspace, int64_t bytes, hipStream_t s);
int activation_slabs(int64_t T, int64_t N);
xtc_status launch_activation_backward(const ActivationArgs &a, hipStream_t s);

int64_t route_workspace(int64_t T, int64_t E);
xtc_status launch_route(const RouteArgs &a, xtc_dtype dtype, void *workspace, hipStream_t s);
xtc_status launch_route_backward(const RouteBackwardArgs &a, xtc_dtype dtype, xtc_dtype out_dtype, hipStream_t s);
xtc_status launch_combine(const CombineArgs &a, xtc_dtype dtype, xtc_dtype r_dtype, xtc_dtype out_dtype, hipStream_t s);
xtc_status launch_combine_backward(const CombineBackwardArgs &a, xtc_dtype dtype, xtc_dtype g_dtype, hipStream_t s);

// The same of a linear layer (1, 2) or its weights' gradient (3): those for rows at any address come first where
// an operand has such, the others then follow (they run on copies).
int linear_kernel(const LinearArgs &a, int kind, int *kernels, int *splits);

// Which of the kernels for aligned rows a product takes (-1: the one for rows at
// any address), and how many there are.  kind: 0 e4m3, 1 bf16 with B [K, N], 2 with
// B [N, K], 3 a weights' gradient.
int grouped_kernel(const GroupedArgs &a, int kind, int *kernels);

}  // namespace xtc

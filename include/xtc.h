/*
 * xtc.h -- C ABI of libxtc.so, the MI355X (gfx950) tiled dense contraction.
 *
 * One function per operator, inputs before outputs, every tensor a raw
 * pointer to contiguous memory (the paper's module ABI, Sec. 4.1, "Module":
 * a function named after the operator that takes the operator's inputs and
 * outputs as contiguous raw pointers).  The schedule is an explicit struct so
 * that schedules can be swept: its fields are the GPU forms of the paper's
 * scheduling primitives (Sec. 3.2, Table 1): strip-mine/tile (block_*,
 * wave_*), vectorize (mfma_*), pack with padding (lds_stages, lds_pad),
 * unroll (unroll_k), parallelize (the workgroup grid) and interchange of the
 * parallel tile loops (raster, xcd_remap).
 *
 * Plain C: no HIP header is needed to use it.  The stream is an opaque
 * hipStream_t passed as void* (NULL = the null stream).
 *
 * Common rules for every entry point
 * ----------------------------------
 * - Tensor pointers are DEVICE pointers, allocated and owned by the caller.
 *   The library allocates nothing, keeps no pointer after it returns and
 *   holds no mutable global state except a thread-local last HIP error code.
 * - Outputs must not overlap inputs (the paper declares its operands
 *   noalias, Fig. 5).  This is not checked.
 * - Every argument and schedule check happens on the host BEFORE any HIP
 *   call, so invalid calls return an error without touching the device.
 * - Kernels are enqueued on `stream`; calls are asynchronous and never
 *   synchronise.  Faults during execution surface at the caller's next
 *   synchronisation on that stream, not in the return value.
 * - The return value is the only error channel.
 * - Element offsets of the matmul and conv2d entry points are 32-bit inside
 *   the kernels: every operand's span
 *   (bytes from its first to its last addressed element) must be at most
 *   0x7FFFFFD0 bytes (2^31 - 48), else XTC_ERR_TOO_LARGE.  Elements
 *   outside an operand (ragged edges, zero padding) are read through a
 *   buffer offset of 0x7FFFFFF0, which this limit keeps past every operand,
 *   so they read as zero.
 */
#ifndef XTC_H
#define XTC_H

#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

/* Element types.  XTC_BF16: inputs are bf16 bit patterns (uint16), products
 * are exact in fp32, accumulation and output are fp32.  XTC_FP8: OCP e4m3
 * (4 exponent and 3 mantissa bits, no infinities, largest value 448), only
 * where an entry point names it. */
typedef enum { XTC_F32 = 0, XTC_BF16 = 1, XTC_FP8 = 2 } xtc_dtype;

typedef enum { XTC_OP_MATMUL = 0, XTC_OP_CONV2D = 1 } xtc_op;

/* What a linear layer applies to its sums (xtc_linear). */
typedef enum {
    XTC_NO_ACTIVATION = 0,
    XTC_RELU = 1,                     /* v < 0 ? 0 : v                        */
    XTC_GELU = 2,                     /* v (1 + erf(v / sqrt 2)) / 2          */
    XTC_GELU_TANH = 3,                /* v (1 + tanh u) / 2, u = sqrt(2/pi)   */
                                      /* (v + 0.044715 v^3)                   */
    XTC_SILU = 4                      /* v / (1 + exp(-v))                    */
} xtc_activation;

typedef enum {
    XTC_OK = 0,
    XTC_ERR_NULL_POINTER = 1,         /* a tensor or output pointer is NULL   */
    XTC_ERR_BAD_SHAPE = 2,            /* negative or inconsistent extents     */
    XTC_ERR_BAD_LEADING_DIM = 3,      /* lda < K, ldb < N or ldc < N (or      */
                                      /* matrices of a family that overlap)   */
    XTC_ERR_BAD_DTYPE = 4,            /* unknown dtype, or not supported here */
    XTC_ERR_BAD_SCHEDULE = 5,         /* illegal field values / combination   */
    XTC_ERR_UNSUPPORTED_SCHEDULE = 6, /* legal but not among compiled ones    */
    XTC_ERR_TOO_LARGE = 7,            /* an operand span above 0x7FFFFFD0     */
                                      /* bytes, or a conv stride/pad/extent   */
                                      /* above 2^30; for the operators on     */
                                      /* blocks, groups and norms see there   */
    XTC_ERR_HIP = 8,                  /* a HIP call failed (see below)        */
    XTC_ERR_MISALIGNED = 9            /* a tensor pointer is not aligned to   */
                                      /* its element size                     */
} xtc_status;

/*
 * Schedule of one contraction C[M,N] = A[M,K] B[K,N] (for conv2d the implicit
 * GEMM: M = OC, N = batch*OH*OW, K = C*R*S; see xtc_conv2d_nchw).
 *
 *  size          sizeof(xtc_sched) as known to the caller (ABI versioning).
 *  block_m/n/k   workgroup tile: the outer strip-mine of M and N (one
 *                workgroup per tile, parallelized over the CUs) and the
 *                K-step staged in LDS per pipeline stage (channels per
 *                stage for the k_order = 2 conv kernels).  Powers of two,
 *                except block_n and wave_n of the k_order = 2 conv kernels
 *                (multiples of 16).
 *  wave_m/n      tile of one 64-lane wavefront inside the workgroup tile
 *                (second strip-mine level); the workgroup has
 *                (block_m/wave_m)*(block_n/wave_n) waves.
 *  mfma_m/n/k    matrix-core instruction tile (the vectorize primitive):
 *                fp32: 32x32x2 or 16x16x4; bf16: 32x32x16 or 16x16x32.
 *  lds_stages    LDS buffers per operand (pack + software pipelining), 1-5;
 *                0 = no LDS staging (the k_split kernels).
 *  lds_pad       LDS row padding in elements (pack with padding against bank
 *                conflicts); -1 selects an XOR-swizzled layout instead.
 *  unroll_k      MFMA k-steps unrolled per LDS stage (0 = the whole stage).
 *  raster        order of the parallel tile loops (interchange): 0 row-major
 *                (N fastest), 1 column-major (M fastest), 2 <= g <= 64
 *                grouped: bands of g tile-rows, walked column by column (a
 *                band taller than the tile grid is the whole grid).  Values
 *                outside 0..64 are XTC_ERR_BAD_SCHEDULE.
 *  xcd_remap     1: renumber workgroups so that each of the 8 XCDs (which
 *                receive workgroups round-robin and each own an L2) works on
 *                one contiguous band of the tile order; 0: hardware order.
 *  k_order       conv2d only (0 for matmul): order of the reduction over
 *                (ic, kh, kw).  0: channel-major, k = (ic*R + kh)*S + kw (the
 *                OIHW weight layout; with block_m = 16, for few output
 *                channels, the workgroup's input patch is staged in LDS
 *                once when it fits, and its two halves of K are reduced by
 *                two groups of waves and added in a fixed order); 1:
 *                tap-major, k = (kh*S + kw)*C + ic
 *                (needs C % 32 == 0, else the channel-major kernel with the
 *                same tiles runs); 2: chunks of channels, and inside a
 *                chunk the R*S taps, with each chunk's input patch staged
 *                once for all taps, for 3x3 stride-1 layers with rows of
 *                about 56 pixels (OW >= 51):
 *                  fp32: chunks of 8, k = ((ic/8)*R*S + kh*S + kw)*8 + ic%8;
 *                  block_n = 256 needs C % 16 == 0 and W + pad_w <= 60;
 *                  block_n = 208 (16x16x4 instructions) needs C % 8 == 0
 *                  and covers at most 208 pixels per workgroup, the count
 *                  chosen per launch so that workgroups split evenly;
 *                  block_n = 416 is the same with two such pixel halves
 *                  per workgroup (8 waves) sharing one input patch;
 *                  other shapes run the tap-major kernel.  lds_pad 0 (the
 *                  patch kernels: 3x3 layers of any stride, padding, row
 *                  length and batch) needs C % 8 == 0 and a patch that fits
 *                  in LDS; other shapes run the tap-major kernel.  Groups
 *                  of waves may share a tile, each reducing every second
 *                  (block_m 64, lds_stages 1) or fourth (block_m 16) stage;
 *                  bf16: chunks of 16, k = ((ic/16)*R*S + kh*S + kw)*16 +
 *                  ic%16.  lds_pad -1 (the kernel for rows of about 56
 *                  pixels) needs C % 16 == 0, even W, pad_w <= 2,
 *                  OW - pad_w <= 60, a 4-byte-aligned X and a 16-byte-
 *                  aligned W; other shapes run a patch kernel, its tile
 *                  chosen by shape.  lds_pad 0 (the patch kernels: 3x3
 *                  layers of any stride, padding, row length and batch)
 *                  needs C % 8 == 0, a 16-byte-aligned W and a patch that
 *                  fits in LDS; other shapes run the channel-major kernel.
 *                  In the patch kernels groups of waves may share a tile,
 *                  each reducing every second or fourth chunk, and their
 *                  sums are added in group order (lds_stages 1: two groups
 *                  for 64x128, four for 32x64; 2: none, two for 32x64);
 *                3: bf16 only, row streaming for 3x3 stride-1 layers of 64
 *                input channels: a workgroup walks down a band of output
 *                rows of one image with all C*R*S weights of its 64 output
 *                channels resident; k = ((kw*4 + ic/16)*3 + kh)*16 + ic%16
 *                per output row.  Needs C == 64, even W, OW % 4 == 0,
 *                OW <= 64, pad_w <= 2, OW + 3 - pad_w <= 63, a 4-byte-
 *                aligned X and 16-byte-aligned W and Y; other shapes run the
 *                k_order 2 kernel.
 *                Results differ only by rounding order.
 *  k_split       waves that share one workgroup tile, each reducing every
 *                k_split-th group of block_k reduction steps (a parallel
 *                split of the reduction for problems with too few tiles to
 *                fill the chip); their partial sums are added in a fixed
 *                order through LDS, so results stay deterministic.  1 = no
 *                split.  With lds_stages = 0 each wave covers the whole
 *                workgroup tile (wave_m = block_m, wave_n = block_n) and
 *                operands go from memory straight to the matrix-core
 *                registers, double-buffered in registers.  With
 *                lds_stages >= 1 (matmul only) k_split groups of
 *                (block_m/wave_m)*(block_n/wave_n) waves each run the
 *                LDS-staged pipeline on every k_split-th K-step of the
 *                tile, each group on its own LDS ring.
 *
 * block_*, wave_*, mfma_*, lds_stages, lds_pad, unroll_k, k_order and k_split
 * select a compiled kernel instance; raster and xcd_remap are run-time choices valid
 * for all.
 */
typedef struct {
    int32_t size;
    int32_t block_m, block_n, block_k;
    int32_t wave_m, wave_n;
    int32_t mfma_m, mfma_n, mfma_k;
    int32_t lds_stages;
    int32_t lds_pad;
    int32_t unroll_k;
    int32_t raster;
    int32_t xcd_remap;
    int32_t k_order;
    int32_t k_split;
} xtc_sched;

/*
 * xtc_matmul -- C = A * B  (paper Sec. 3.1, Fig. 2: C[i][j] accumulates
 * A[i][k]*B[k][j] over k; here C is overwritten, i.e. accumulation starts
 * from zero).
 *
 *  M, N, K   extents, >= 0.  M == 0 or N == 0: no-op returning XTC_OK.
 *            K == 0: C[0:M, 0:N] is set to zero.
 *  A         device, row-major M x K with row stride lda >= max(K,1)
 *            (elements); fp32 (XTC_F32) or bf16 bits (XTC_BF16).
 *  B         device, row-major K x N with row stride ldb >= max(N,1).
 *  C         device, fp32, row-major M x N with row stride ldc >= max(N,1).
 *            Only C[i*ldc + j] for i < M, j < N is written; columns
 *            N <= j < ldc are never touched.
 *  dtype     XTC_F32 or XTC_BF16 (applies to A and B; C is always fp32).
 *            A, B and C are aligned to their element size (4 bytes fp32,
 *            2 bytes bf16); any row stride is accepted.
 *  sched     NULL selects xtc_default_schedule(); otherwise must pass
 *            xtc_sched_check().
 *  stream    hipStream_t or NULL.
 * Errors: XTC_ERR_NULL_POINTER (A, B or C NULL while M, N > 0),
 * XTC_ERR_BAD_SHAPE (negative extent), XTC_ERR_BAD_LEADING_DIM,
 * XTC_ERR_BAD_DTYPE, XTC_ERR_MISALIGNED (a pointer not aligned to its
 * element size), XTC_ERR_BAD_SCHEDULE, XTC_ERR_UNSUPPORTED_SCHEDULE,
 * XTC_ERR_TOO_LARGE, XTC_ERR_HIP (launch failed).
 */
xtc_status xtc_matmul(int64_t M, int64_t N, int64_t K,
                      const void *A, int64_t lda,
                      const void *B, int64_t ldb,
                      float *C, int64_t ldc,
                      xtc_dtype dtype, const xtc_sched *sched, void *stream);

/*
 * xtc_conv2d_nchw -- 2-D convolution (the paper's conv2d operator, Sec. 3.1)
 * read as zero-padded cross-correlation without dilation, groups or bias:
 *   Y[n][oc][oh][ow] = sum_{ic<C, kh<R, kw<S}
 *        X[n][ic][oh*stride_h - pad_h + kh][ow*stride_w - pad_w + kw]
 *        * Wt[oc][ic][kh][kw],
 * input positions outside [0,H) x [0,W) contributing zero, with
 *   OH = (H + 2*pad_h - R)/stride_h + 1,  OW = (W + 2*pad_w - S)/stride_w + 1.
 * Computed as an implicit GEMM (no im2col buffer): M = OC, N = N*OH*OW,
 * K = C*R*S, reduced in the order the schedule's k_order selects.
 *
 *  X    device, NCHW contiguous; Wt device, OIHW contiguous; both fp32
 *       (XTC_F32) or both bf16 bit patterns (XTC_BF16, products exact in
 *       fp32, fp32 accumulation).
 *  Y    device, N x OC x OH x OW contiguous fp32 (overwritten).
 *  X, Wt and Y are aligned to their element size (else XTC_ERR_MISALIGNED).
 *  N, C, H, W, OC, R, S >= 1 except that N == 0 or OC == 0 is a no-op;
 *  stride >= 1, pad >= 0, OH >= 1 and OW >= 1, else XTC_ERR_BAD_SHAPE.
 *  stride_h, stride_w, pad_h, pad_w, H, W, H + 2*pad_h and W + 2*pad_w are
 *  at most 2^30 (input coordinates stay in 32-bit arithmetic), else
 *  XTC_ERR_TOO_LARGE.
 *  dtype XTC_F32 or XTC_BF16 (else XTC_ERR_BAD_DTYPE); each reduces in
 *  the order its schedule's k_order selects (bf16: 0, 2 or 3).
 *  sched NULL selects the default conv schedule's kernel, with three
 *  exceptions by shape: large fp32 3x3 layers of whole 8-channel groups run
 *  the patch, halo, tap-major or k-table kernel whose tiles share the CUs
 *  best; fp32 layers of 17 to 32 output channels and a short reduction the
 *  16-channel, patch or 64x64 tiles likewise; and pointwise layers
 *  (1x1, stride 1, no padding), which the matmul kernels compute per image,
 *  with xtc_default_schedule's matmul rules, where that is the faster route
 *  (not for many images smaller than a tile, nor for bf16 layers of fewer than
 *  32 channels, or of up to 64 whose images do not start on 16 bytes; fp32
 *  layers of up to 16 output channels take tiles that add as many partial sums
 *  as the conv kernel, from 64 channels on).
 * Errors as for xtc_matmul; XTC_ERR_TOO_LARGE also when C*R*S exceeds the
 * kernel's k-offset table capacity (xtc_conv_max_k()).
 */
xtc_status xtc_conv2d_nchw(int64_t N, int64_t C, int64_t H, int64_t W,
                           int64_t OC, int64_t R, int64_t S,
                           int64_t stride_h, int64_t stride_w,
                           int64_t pad_h, int64_t pad_w,
                           const void *X, const void *Wt, float *Y,
                           xtc_dtype dtype, const xtc_sched *sched, void *stream);

/*
 * xtc_matmul_relu, xtc_conv2d_nchw_relu -- the contraction followed by its
 * consumer relu, fused into the epilogue (the paper's matmul+relu graph,
 * Sec. 5.2, Fig. 9, and its "fusion of consumer", Sec. 3.2): every output
 * element is written once, as relu(v) = (v < 0 ? 0 : v) of the value v that
 * xtc_matmul / xtc_conv2d_nchw would write (a NaN stays NaN, -0.0 stays
 * -0.0).  Arguments, layouts, ownership, schedules and errors are exactly
 * those of xtc_matmul / xtc_conv2d_nchw; the same kernel instances run, so
 * no extra pass over the output and no extra memory traffic is added.
 */
xtc_status xtc_matmul_relu(int64_t M, int64_t N, int64_t K,
                           const void *A, int64_t lda,
                           const void *B, int64_t ldb,
                           float *C, int64_t ldc,
                           xtc_dtype dtype, const xtc_sched *sched, void *stream);

xtc_status xtc_conv2d_nchw_relu(int64_t N, int64_t C, int64_t H, int64_t W,
                                int64_t OC, int64_t R, int64_t S,
                                int64_t stride_h, int64_t stride_w,
                                int64_t pad_h, int64_t pad_w,
                                const void *X, const void *Wt, float *Y,
                                xtc_dtype dtype, const xtc_sched *sched, void *stream);

/*
 * Operators around the products of a transformer block: the norm in front of
 * them, products of 8-bit operands whose values share scales, and products of
 * rows that belong to different matrices (the experts of a mixture).
 *
 * Limits of these entry points: extents at most 0x7FFFFF00, row strides at most
 * 2^30 elements, matrices of a family at most 2^50 elements apart, and a launch
 * of fewer than 2^24 workgroups, else XTC_ERR_TOO_LARGE.  Offsets are 64-bit:
 * operands may exceed 2^31 bytes.  Every row stride is at least the row's
 * length, else XTC_ERR_BAD_LEADING_DIM.  Rows may start at any element boundary;
 * 16-byte aligned rows of a multiple of 16 bytes run the faster kernels.
 *
 * 8-bit operands.  A matrix of e4m3 values has fp32 scales S for blocks of 128
 * consecutive values of a row: value (i, j) stands for Q[i][j] * S[i][j/128], or
 * S[i/128][j/128] where 128 rows share scales; the last blocks may be cut.
 */

/*
 * xtc_rmsnorm -- root-mean-square norm of each row of X + R:
 *   h = X + R (fp32), rstd = 1 / sqrt(sum_j h_j^2 / D + eps),
 *   Y_j = W_j * h_j * rstd, rounded once.
 *
 *  T, D       rows and columns, >= 0; either 0 is a no-op (with D 0, whose
 *             means are 0/0, rstd is left as it is).
 *  X, R       device, dtype (XTC_F32 or XTC_BF16), row strides ldx, ldr.  R NULL:
 *             nothing is added.
 *  W          device, D values of w_dtype: dtype or XTC_F32.
 *  eps        >= 0, else XTC_ERR_BAD_SHAPE.
 *  Y          device, out_dtype: dtype, or XTC_FP8 with the scales S (fp32,
 *             T x ceil(D/128), row stride lds): S = max(amax / 448, 2^-126), amax
 *             the largest finite magnitude of the block's 128 unrounded outputs,
 *             each then divided by S and rounded to nearest even; an output
 *             that is not finite becomes e4m3's NaN.
 *  H          device, dtype: h rounded once (the residual of the next norm), or
 *             NULL.  Needs R.
 *  rstd       device, T fp32 values for the gradient, or NULL.
 * Errors: XTC_ERR_BAD_DTYPE, XTC_ERR_BAD_SHAPE, XTC_ERR_TOO_LARGE,
 * XTC_ERR_BAD_LEADING_DIM, XTC_ERR_NULL_POINTER, XTC_ERR_MISALIGNED, XTC_ERR_HIP.
 */
xtc_status xtc_rmsnorm(int64_t T, int64_t D, const void *X, int64_t ldx,
                       const void *R, int64_t ldr, const void *W, float eps,
                       void *Y, int64_t ldy, float *S, int64_t lds,
                       void *H, int64_t ldh, float *rstd,
                       xtc_dtype dtype, xtc_dtype w_dtype, xtc_dtype out_dtype, void *stream);

/*
 * xtc_rmsnorm_backward -- the norm's gradient.  X is what was normalised (H
 * where a residual was added) and rstd what xtc_rmsnorm kept; with
 * xh = X * rstd and g = DY * W,
 *   DX = rstd * (g - xh * sum_j(g_j xh_j) / D) + DR,  DW_j = sum_t DY_tj xh_tj.
 * DX is the gradient of both summands of X + R.
 *
 *  DY, X, DX  device, dtype, row strides lddy, ldx, lddx.
 *  DR         gradient that reaches the sum from elsewhere (row stride lddr), or
 *             NULL.
 *  DW         device, D fp32 values (overwritten; zeros when T == 0).
 *  workspace  device, workspace_bytes >= xtc_rmsnorm_backward_workspace(T, D),
 *             16-byte aligned, written by the call; too small is
 *             XTC_ERR_BAD_SHAPE.
 * Sums are fp32 in an order that depends on T and D alone.
 * Errors as for xtc_rmsnorm.
 */
xtc_status xtc_rmsnorm_backward(int64_t T, int64_t D, const void *DY, int64_t lddy,
                                const void *X, int64_t ldx, const void *W, const float *rstd,
                                const void *DR, int64_t lddr, void *DX, int64_t lddx, float *DW,
                                void *workspace, int64_t workspace_bytes,
                                xtc_dtype dtype, xtc_dtype w_dtype, void *stream);

/* Bytes of workspace for T rows of D columns; -1 for extents outside the limits.  Pure host function. */
int64_t xtc_rmsnorm_backward_workspace(int64_t T, int64_t D);

/*
 * xtc_layernorm -- layer norm of each row of X + R:
 *   h = X + R (fp32), mean = sum_j h_j / D, rstd = 1 / sqrt(sum_j (h_j - mean)^2 / D + eps),
 *   Y_j = W_j * (h_j - mean) * rstd + B_j, rounded once.
 * B (device, D values of w_dtype) may be NULL: nothing is added.  mean and rstd are
 * device, T fp32 values each for the gradient, or NULL.  All else, 8-bit outputs
 * and errors among it, as for xtc_rmsnorm; sums are fp32.
 */
xtc_status xtc_layernorm(int64_t T, int64_t D, const void *X, int64_t ldx,
                         const void *R, int64_t ldr, const void *W, const void *B, float eps,
                         void *Y, int64_t ldy, float *S, int64_t lds,
                         void *H, int64_t ldh, float *mean, float *rstd,
                         xtc_dtype dtype, xtc_dtype w_dtype, xtc_dtype out_dtype, void *stream);

/*
 * xtc_layernorm_backward -- the layer norm's gradient.  X is what was normalised and
 * mean, rstd what xtc_layernorm kept; with xh = (X - mean) * rstd and g = DY * W,
 *   DX = rstd * (g - sum_j g_j / D - xh * sum_j(g_j xh_j) / D) + DR,
 *   DW_j = sum_t DY_tj xh_tj,  DB_j = sum_t DY_tj.
 * DB: device, D fp32 values, like DW.  All else as for xtc_rmsnorm_backward, with
 * xtc_layernorm_backward_workspace(T, D).
 */
xtc_status xtc_layernorm_backward(int64_t T, int64_t D, const void *DY, int64_t lddy,
                                  const void *X, int64_t ldx, const void *W,
                                  const float *mean, const float *rstd,
                                  const void *DR, int64_t lddr, void *DX, int64_t lddx,
                                  float *DW, float *DB, void *workspace, int64_t workspace_bytes,
                                  xtc_dtype dtype, xtc_dtype w_dtype, void *stream);

/* Bytes of workspace for T rows of D columns; -1 for extents outside the limits.  Pure host function. */
int64_t xtc_layernorm_backward_workspace(int64_t T, int64_t D);

/*
 * xtc_quantize_fp8 -- X [M, K] (dtype, row stride ldx) as e4m3 values Q (row
 * stride ldq) and scales S (row stride lds): one for each block_rows x 128
 * values, block_rows 1 (activations) or 128 (weights), else XTC_ERR_BAD_SHAPE.
 * S = max(amax / 448, 2^-126) over the block's finite magnitudes, Q = X / S
 * rounded to nearest even; what is not finite becomes NaN.  M or K 0: no-op.
 * Errors as for xtc_rmsnorm.
 */
xtc_status xtc_quantize_fp8(int64_t M, int64_t K, const void *X, int64_t ldx, int64_t block_rows,
                            void *Q, int64_t ldq, float *S, int64_t lds,
                            xtc_dtype dtype, void *stream);

/*
 * xtc_matmul_fp8 -- C = A * B^T of block-scaled e4m3 operands:
 *   C[m][n] = sum_b SA[m][b] SB[n/128][b] sum_{k in block b} A[m][k] B[n][k],
 * the inner sums and the outer one in fp32, rounded once into C.  For XTC_BF16
 * the inner sums are the 8-bit matrix instructions': of eight consecutive
 * products, what lies more than 13 binary places below the largest is cut off,
 * 1.5e-5 of a typical result, a hundredth of its rounding.  Where large products
 * cancel it can be 2^-10 of the largest of each eight, whatever is left: sums that
 * may cancel are for XTC_F32.  A block's two scales are multiplied first, in
 * fp32: where that product is no normal number (below 2^-126, or an overflow), so
 * is the result less exact, or not finite.
 *
 *  A   e4m3 M x K, row stride lda; SA its scales, one per row and 128 k, row
 *      stride ldsa.
 *  B   e4m3 N x K (a row holds the weights of one output), row stride ldb; SB
 *      its scales, one per 128 rows and 128 k, row stride ldsb.
 *  C   out_dtype XTC_F32 or XTC_BF16, M x N, row stride ldc.
 *  relu  nonzero: C holds v < 0 ? 0 : v (a NaN stays NaN).
 * M or N 0 is a no-op; K 0 gives zeros.  Errors as for xtc_rmsnorm.
 */
xtc_status xtc_matmul_fp8(int64_t M, int64_t N, int64_t K,
                          const void *A, int64_t lda, const float *SA, int64_t ldsa,
                          const void *B, int64_t ldb, const float *SB, int64_t ldsb,
                          void *C, int64_t ldc, xtc_dtype out_dtype, int32_t relu, void *stream);

/*
 * xtc_linear -- a linear layer and what follows it:
 *   z = A * B + bias,  C = act(z) + R,
 * sums and all of that in fp32, z and C rounded once each.
 *
 *  A      bf16 (dtype XTC_BF16, else XTC_ERR_BAD_DTYPE) T x K, row stride lda.
 *  B      bf16 K x N, row stride ldb, or N x K where transpose_b is nonzero (the
 *         gradient of A is the product of z's gradient with the same B and the
 *         other transpose_b).
 *  bias   device, N values of bias_dtype (XTC_F32 or XTC_BF16), or NULL.
 *  R      device, T x N of r_dtype (XTC_F32 or XTC_BF16), row stride ldr, or NULL.
 *  activation  an xtc_activation, else XTC_ERR_BAD_SHAPE.
 *  C      device, out_dtype (XTC_F32 or XTC_BF16) T x N, row stride ldc.  It may be
 *         R itself (ldc == ldr, out_dtype == r_dtype).
 *  Z      device, z in out_dtype for the activation's gradient, row stride ldz, or
 *         NULL.
 *  workspace  device, workspace_bytes >= xtc_linear_workspace() of the same operands
 *         (0 for many sizes: NULL is fine then), 16-byte aligned, written by the
 *         call; too small is XTC_ERR_BAD_SHAPE.  Calls that may run at the same
 *         time need one each.
 * T or N 0 is a no-op; K 0 gives act(bias) + R.  The order of a sum depends on T, N,
 * K, transpose_b and on which rows are 16-byte aligned.  Errors as for xtc_rmsnorm.
 */
xtc_status xtc_linear(int64_t T, int64_t N, int64_t K, const void *A, int64_t lda,
                      const void *B, int64_t ldb, int32_t transpose_b,
                      const void *bias, xtc_dtype bias_dtype,
                      const void *R, int64_t ldr, xtc_dtype r_dtype, int32_t activation,
                      void *C, int64_t ldc, void *Z, int64_t ldz,
                      void *workspace, int64_t workspace_bytes,
                      xtc_dtype dtype, xtc_dtype out_dtype, void *stream);

/* Bytes of workspace, 640 MiB at most; -1 for extents outside the limits.  Pure host function:
 * of the pointers and strides it takes the alignment (rows off 16 bytes may be copied first,
 * where the copies take 512 MiB at most; the sums of a divided reduction take the rest). */
int64_t xtc_linear_workspace(int64_t T, int64_t N, int64_t K, const void *A, int64_t lda,
                             const void *B, int64_t ldb, int32_t transpose_b);

/*
 * xtc_linear_wgrad -- the gradient of a linear layer's B: DB = A^T * DY (zeros when
 * T == 0), K x N of out_dtype (XTC_F32 or XTC_BF16), row stride lddb.  A is T x K, DY
 * (z's gradient) T x N, both bf16.  Of a B that is N x K it is the same call with A
 * and DY exchanged.  workspace: xtc_linear_wgrad_workspace() bytes, as above.
 */
xtc_status xtc_linear_wgrad(int64_t T, int64_t N, int64_t K, const void *A, int64_t lda,
                            const void *DY, int64_t lddy, void *DB, int64_t lddb,
                            void *workspace, int64_t workspace_bytes,
                            xtc_dtype dtype, xtc_dtype out_dtype, void *stream);

/* Bytes of workspace, as above. */
int64_t xtc_linear_wgrad_workspace(int64_t T, int64_t N, int64_t K, const void *A, int64_t lda,
                                   const void *DY, int64_t lddy);

/*
 * xtc_activation_backward -- the gradients of a linear layer's z and bias:
 *   DZ = DY * act'(Z), DB_j = sum_t DY_tj act'(Z_tj),
 * the product in fp32, DZ rounded once to bf16 (what xtc_linear and
 * xtc_linear_wgrad take) and DB summed, in fp32, before that rounding.
 *
 *  DY, Z  device, T x N of dy_dtype and z_dtype (XTC_F32 or XTC_BF16 each), row
 *         strides lddy and ldz.  With XTC_NO_ACTIVATION Z and what describes it are ignored.
 *  DZ     device, bf16 T x N, row stride lddz.
 *  DB     device, N fp32 values (zeros when T == 0), or NULL.
 *  workspace  xtc_activation_backward_workspace(T, N) bytes, as above; without DB
 *         none is needed.
 * Sums are taken in an order that depends on T and N alone.
 */
xtc_status xtc_activation_backward(int64_t T, int64_t N, const void *DY, int64_t lddy, xtc_dtype dy_dtype,
                                   const void *Z, int64_t ldz, xtc_dtype z_dtype, int32_t activation,
                                   void *DZ, int64_t lddz, float *DB,
                                   void *workspace, int64_t workspace_bytes, void *stream);

/* Bytes of workspace; -1 for extents outside the limits.  Pure host function. */
int64_t xtc_activation_backward_workspace(int64_t T, int64_t N);

/*
 * xtc_matmul_grouped -- products of the rows of A with the matrix of their
 * group: C[i] = A[i] * B[g] for the rows i of group g.
 *
 *  G, T   groups (>= 1, else XTC_ERR_BAD_SHAPE) and rows of A.
 *  ends   device, G values: group g holds the rows from ends[g-1] (0 for the
 *         first) to ends[g]; they ascend to at most T.  A value below an earlier
 *         one makes an empty group, one above T counts as T.  Rows from
 *         ends[G-1] to T belong to no group: C is zero there.
 *  A      bf16 (dtype XTC_BF16, else XTC_ERR_BAD_DTYPE) T x K, row stride lda.
 *  B      G matrices stride_b elements apart, each K x N with row stride ldb,
 *         or N x K where transpose_b is nonzero (the gradient of A is the
 *         product of C's gradient with the same B and the other transpose_b).
 *  C      out_dtype XTC_F32 or XTC_BF16, T x N, row stride ldc; fp32 sums,
 *         rounded once.
 *  relu   as for xtc_matmul_fp8.
 * The sizes of the groups stay on the device.  Errors as for xtc_rmsnorm.
 */
xtc_status xtc_matmul_grouped(int64_t G, int64_t T, int64_t N, int64_t K,
                              const void *A, int64_t lda,
                              const void *B, int64_t ldb, int64_t stride_b, int32_t transpose_b,
                              const int32_t *ends, void *C, int64_t ldc,
                              xtc_dtype dtype, xtc_dtype out_dtype, int32_t relu, void *stream);

/*
 * xtc_matmul_grouped_wgrad -- the gradient of B: DB[g] = A_g^T * DY_g over the
 * rows of group g (zeros for an empty one).  A is T x K, DY T x N, both bf16;
 * DB holds G matrices K x N of out_dtype (XTC_F32 or XTC_BF16) stride_db
 * elements apart, row stride lddb.  ends and errors as for xtc_matmul_grouped.
 */
xtc_status xtc_matmul_grouped_wgrad(int64_t G, int64_t T, int64_t N, int64_t K,
                                    const void *A, int64_t lda, const void *DY, int64_t lddy,
                                    const int32_t *ends, void *DB, int64_t lddb, int64_t stride_db,
                                    xtc_dtype dtype, xtc_dtype out_dtype, void *stream);

/*
 * xtc_matmul_grouped_fp8 -- xtc_matmul_grouped of block-scaled e4m3 operands
 * (see xtc_matmul_fp8): B holds G matrices N x K stride_b elements apart, SB
 * their scales stride_sb values apart.
 */
xtc_status xtc_matmul_grouped_fp8(int64_t G, int64_t T, int64_t N, int64_t K,
                                  const void *A, int64_t lda, const float *SA, int64_t ldsa,
                                  const void *B, int64_t ldb, int64_t stride_b,
                                  const float *SB, int64_t ldsb, int64_t stride_sb,
                                  const int32_t *ends, void *C, int64_t ldc,
                                  xtc_dtype out_dtype, int32_t relu, void *stream);

/*
 * xtc_route_experts -- the router of a mixture of experts: which experts T tokens
 * go to, with which weights, and where their rows lie when sorted by expert, as
 * the grouped products take them.
 *
 *  E, top     experts (1 to 1024) and how many a token chooses (1 to 16, at most E);
 *             T * top at most 0x7FFFFF00.
 *  scores     device, dtype (XTC_F32 or XTC_BF16) T x E, row stride lds.  An expert
 *             at -inf has the weight 0, and is chosen only where fewer than top
 *             others are left; a NaN counts as above every number.
 *  mask       device, T bytes, 0 for a token that goes nowhere (padding), or NULL.
 *  expert     T x top: the experts of each token, the highest score first, of equal
 *             scores the lowest index; -1 for a masked token.
 *  p          T x top fp32: the softmax of the chosen scores; 0 for a masked token
 *             and for one whose scores are all -inf.
 *  row        T x top: the place of each choice among the rows sorted by expert, those
 *             of an expert in the order of their tokens; -1 for a masked token.
 *  token      T * top: the token of each of these rows; -1 behind the last one.
 *  counts, ends  E each: the rows of each expert, and where they end.
 *  loss       one fp32: the balance loss E / (top n^2) sum_e counts_e sum_t q_te, q the
 *             softmax over all experts (0 for a row of -inf), n the tokens that are not
 *             masked; 0 without any.  It is 1 where all experts are chosen equally.
 *  workspace  xtc_route_experts_workspace(T, E) bytes (0 for few tokens: NULL is fine
 *             then), 16-byte aligned, written by the call; too small is XTC_ERR_BAD_SHAPE.
 * All arrays but scores are contiguous.  Outputs are the same bits in every call.  With
 * T 0 counts, ends and loss are zeros.  Errors as for xtc_rmsnorm.
 */
xtc_status xtc_route_experts(int64_t T, int64_t E, int64_t top, const void *scores, int64_t lds,
                             const uint8_t *mask, int32_t *expert, float *p, int32_t *row,
                             int32_t *token, int32_t *counts, int32_t *ends, float *loss,
                             void *workspace, int64_t workspace_bytes,
                             xtc_dtype dtype, void *stream);

/* Bytes of workspace; -1 for extents outside the limits.  Pure host function. */
int64_t xtc_route_experts_workspace(int64_t T, int64_t E);

/*
 * xtc_route_experts_backward -- the gradient of the scores, from DP (T x top fp32, the
 * gradient of p; NULL: zeros) and dloss, that of the balance loss:
 *   DS = dloss E / (top n^2) q_e (counts_e - sum_i counts_i q_i), and at the chosen
 *        experts p_j (DP_j - sum_i p_i DP_i) added; zeros for a masked token.
 * scores, expert, p and counts as xtc_route_experts took and gave them (n is the sum of
 * counts over top).  DS: device, out_dtype (XTC_F32 or XTC_BF16) T x E, row stride
 * ldds.  Errors as for xtc_rmsnorm.
 */
xtc_status xtc_route_experts_backward(int64_t T, int64_t E, int64_t top, const float *DP,
                                      const void *scores, int64_t lds, const int32_t *expert,
                                      const float *p, const int32_t *counts, float dloss,
                                      void *DS, int64_t ldds,
                                      xtc_dtype dtype, xtc_dtype out_dtype, void *stream);

/*
 * xtc_combine_experts -- the experts' rows back at their tokens:
 *   C[t] = RES[t] + sum_j p[t][j] * rows[row[t][j]], in fp32, over j in its order.
 *
 *  rows   device, dtype (XTC_F32 or XTC_BF16) R x D, row stride ldrows.
 *  row    device, T x top, contiguous.  What lies outside 0 .. R - 1 (-1: a masked
 *         choice) counts as a row of zeros.
 *  p      device, T x top fp32, contiguous, or NULL: ones (the gradient of rows that
 *         were copied to their experts).
 *  RES    device, T x D of r_dtype (XTC_F32 or XTC_BF16), row stride ldr, or NULL.
 *  C      device, out_dtype (XTC_F32 or XTC_BF16) T x D, row stride ldc.
 * T or D 0 is a no-op; top 0 gives RES.  T * top at most 0x7FFFFF00.  Errors as for
 * xtc_rmsnorm.
 */
xtc_status xtc_combine_experts(int64_t T, int64_t top, int64_t D, int64_t R,
                               const void *rows, int64_t ldrows, const int32_t *row, const float *p,
                               const void *RES, int64_t ldr, xtc_dtype r_dtype,
                               void *C, int64_t ldc, xtc_dtype dtype, xtc_dtype out_dtype, void *stream);

/*
 * xtc_combine_experts_backward -- its gradients, for T * top rows each of which is one
 * choice's at most (as xtc_route_experts gives them):
 *   DROWS[row[t][j]] = p[t][j] * DOUT[t],  DP[t][j] = sum_d DOUT[t][d] rows[row[t][j]][d].
 * Rows that belong to no token (token -1) are zeros in DROWS, DP of a masked choice is 0.
 * DOUT: T x D of dout_dtype, row stride lddo; rows and DROWS of dtype (XTC_F32 or
 * XTC_BF16 each); DP T x top fp32.  top >= 1, else XTC_ERR_BAD_SHAPE; with D 0 DP is
 * zeros.  Errors as for xtc_rmsnorm.
 */
xtc_status xtc_combine_experts_backward(int64_t T, int64_t top, int64_t D, const void *DOUT, int64_t lddo,
                                        xtc_dtype dout_dtype, const void *rows, int64_t ldrows,
                                        const int32_t *row, const int32_t *token, const float *p,
                                        void *DROWS, int64_t lddr, float *DP,
                                        xtc_dtype dtype, void *stream);

/*
 * xtc_default_schedule -- the schedule used when sched == NULL, chosen from
 * the problem shape (the paper's default_schedule of an exploration
 * strategy, Sec. 5.2).  For op == XTC_OP_CONV2D pass the implicit-GEMM
 * extents.  Pure host function.  Errors: XTC_ERR_NULL_POINTER (out NULL),
 * XTC_ERR_BAD_DTYPE, XTC_ERR_BAD_SHAPE.
 */
xtc_status xtc_default_schedule(xtc_op op, xtc_dtype dtype,
                                int64_t M, int64_t N, int64_t K, xtc_sched *out);

/*
 * xtc_sched_check -- XTC_OK if `s` can run op/dtype: its fields are legal
 * (XTC_ERR_BAD_SCHEDULE otherwise) and they name a compiled instance
 * (XTC_ERR_UNSUPPORTED_SCHEDULE otherwise).  This is the membership test of
 * the design space a scheduling strategy samples from (Sec. 5.2: a strategy
 * defines a design space over a scheduling template and turns a sample into
 * a schedule); the fields are the primitives of Table 1 (Sec. 3.2).
 * Pure host function; `s` is only read.  Errors: XTC_ERR_NULL_POINTER (s
 * NULL), XTC_ERR_BAD_DTYPE, XTC_ERR_BAD_SCHEDULE (also an unknown op),
 * XTC_ERR_UNSUPPORTED_SCHEDULE.
 */
xtc_status xtc_sched_check(xtc_op op, xtc_dtype dtype, const xtc_sched *s);

/*
 * xtc_sched_list -- the compiled part of the design space (Sec. 5.2: the
 * grid a strategy samples from): writes up to `cap` compiled schedules for
 * op/dtype into the caller-owned array `out` (may be NULL when cap is 0;
 * each entry has raster = 0, xcd_remap = 1) and returns how many exist in
 * total (call with cap = 0 to size the array).  Combined with every raster
 * and xcd_remap value they span the schedules an exploration can sample.
 * Returns -1 for an unknown op/dtype.  Pure host function.
 */
int32_t xtc_sched_list(xtc_op op, xtc_dtype dtype, xtc_sched *out, int32_t cap);

/*
 * xtc_sched_occupancy -- how many workgroups of the kernel instance `s`
 * names one CU holds at once (an input of the per-schedule traffic model
 * evaluated against hardware counters, the GPU form of the cache-model
 * study of Sec. 6.3: the tiles resident together decide what the caches
 * share) (the hardware limit set by the kernel's
 * registers, LDS and threads), for reduction length K (matmul: K; conv2d:
 * C*R*S, which sizes the conv kernels' LDS k-offset table).  For a conv
 * tap-major instance the figure is that of the tap-major kernel itself, not
 * of the channel-major kernel it falls back to when C % 32 != 0.  The LDS of
 * the patch kernels (k_order 2, lds_pad 0) holds a tile's input patch, which
 * depends on the layer: their figure is that of a 28x28 image at stride 1 and
 * padding 1, whatever K; longer rows, strides or a batch may leave fewer.  Queries
 * the current HIP device; enqueues nothing.  Errors: XTC_ERR_NULL_POINTER,
 * the codes of xtc_sched_check, XTC_ERR_BAD_SHAPE (K < 0),
 * XTC_ERR_TOO_LARGE (conv K above xtc_conv_max_k(), or K > 2^30),
 * XTC_ERR_HIP.
 */
xtc_status xtc_sched_occupancy(xtc_op op, xtc_dtype dtype, int64_t K,
                               const xtc_sched *s, int32_t *wg_per_cu);

/*
 * xtc_status_str -- static, NUL-terminated description of a status code, for
 * the harness that reports why a generated operator could not run (Sec. 4.2:
 * the Executor validates results, the Evaluator runs the code and collects
 * metrics).  Never NULL ("unknown status" for a value outside the enum); the
 * string is owned by the library and must not be freed.
 */
const char *xtc_status_str(xtc_status s);

/*
 * xtc_last_hip_error -- hipError_t value of the last failed HIP call made by
 * this thread inside the library, 0 if none (the detail behind XTC_ERR_HIP,
 * for the harness of Sec. 4.2).  Thread-local; not reset by later
 * successful calls.
 */
int32_t xtc_last_hip_error(void);

/*
 * xtc_conv_max_k -- largest reduction length C*R*S that xtc_conv2d_nchw
 * accepts (the capacity of the conv kernels' k-offset table; the conv2d
 * operator of Sec. 3.1 lowered to an implicit GEMM).  Pure host function.
 */
int64_t xtc_conv_max_k(void);

/*
 * xtc_version -- library version, major*10000 + minor*100 + patch, so that a
 * caller loading the module (Sec. 4.1, "Module": a shared library loaded at
 * run time) can check the ABI it binds to.  Pure host function.
 */
int32_t xtc_version(void);

#ifdef __cplusplus
}
#endif

#endif /* XTC_H */

// Host side of the 8-bit, grouped and normalisation operators of
// include/xtc.h: argument checks (before any HIP call) and the launch on the
// caller's stream.
#include "operators.h"

namespace {

using namespace xtc;

constexpr int64_t kMostExtent = 0x7FFFFF00;   // rows and columns: 32-bit counts, tiles past the end included

bool aligned_to(const void *p, int64_t bytes) { return (reinterpret_cast<uintptr_t>(p) & (uintptr_t)(bytes - 1)) == 0; }
bool known(xtc_dtype t) { return t == XTC_F32 || t == XTC_BF16; }
int64_t size_of(xtc_dtype t) { return t == XTC_F32 ? 4 : t == XTC_BF16 ? 2 : 1; }
int64_t least(int64_t extent) { return extent > 1 ? extent : 1; }
int64_t scale_blocks(int64_t k) { return k / kScaleBlock + (k % kScaleBlock != 0); }

// Row strides are at most 2^30 elements, matrices of a family 2^50 apart: offsets stay in 64 bits.
constexpr int64_t kMostStride = int64_t(1) << 30;

}  // namespace

extern "C" {

xtc_status xtc_rmsnorm(int64_t T, int64_t D, const void *X, int64_t ldx, const void *R, int64_t ldr, const void *W,
                       float eps, void *Y, int64_t ldy, float *S, int64_t lds, void *H, int64_t ldh, float *rstd,
                       xtc_dtype dtype, xtc_dtype w_dtype, xtc_dtype out_dtype, void *stream) {
    const bool quantize = out_dtype == XTC_FP8;
    if (!known(dtype) || (w_dtype != dtype && w_dtype != XTC_F32) || (!quantize && out_dtype != dtype))
        return XTC_ERR_BAD_DTYPE;
    if (T < 0 || D < 0 || !(eps >= 0.f)) return XTC_ERR_BAD_SHAPE;
    if (T == 0 || D == 0) return XTC_OK;
    if (T > kMostExtent || D > kMostExtent || ldx > kMostStride || ldy > kMostStride || (R && ldr > kMostStride) ||
        (H && ldh > kMostStride) || (quantize && lds > kMostStride))
        return XTC_ERR_TOO_LARGE;
    if (ldx < D || ldy < D || (R && ldr < D) || (H && ldh < D) || (quantize && lds < scale_blocks(D)))
        return XTC_ERR_BAD_LEADING_DIM;
    if (!X || !W || !Y || (quantize && !S) || (H && !R)) return XTC_ERR_NULL_POINTER;
    const int64_t e = size_of(dtype);
    if (!aligned_to(X, e) || !aligned_to(R, e) || !aligned_to(H, e) || !aligned_to(W, size_of(w_dtype)) ||
        !aligned_to(Y, size_of(out_dtype)) || !aligned_to(S, 4) || !aligned_to(rstd, 4))
        return XTC_ERR_MISALIGNED;
    NormArgs a;
    a.T = T; a.D = (int)D;
    a.X = X; a.ldx = ldx; a.R = R; a.ldr = ldr;
    a.W = W; a.w_f32 = w_dtype == XTC_F32; a.eps = eps;
    a.Y = Y; a.ldy = ldy; a.S = S; a.lds = lds;
    a.H = H; a.ldh = ldh; a.rstd = rstd;
    return launch_rmsnorm(a, dtype, quantize, static_cast<hipStream_t>(stream));
}

int64_t xtc_rmsnorm_backward_workspace(int64_t T, int64_t D) {
    if (T < 0 || D < 0 || T > kMostExtent || D > kMostExtent) return -1;
    return 4 * norm_backward_slabs(T, D) * D;
}

xtc_status xtc_rmsnorm_backward(int64_t T, int64_t D, const void *DY, int64_t lddy, const void *X, int64_t ldx,
                                const void *W, const float *rstd, const void *DR, int64_t lddr, void *DX, int64_t lddx,
                                float *DW, void *workspace, int64_t workspace_bytes, xtc_dtype dtype,
                                xtc_dtype w_dtype, void *stream) {
    if (!known(dtype) || (w_dtype != dtype && w_dtype != XTC_F32)) return XTC_ERR_BAD_DTYPE;
    if (T < 0 || D < 0) return XTC_ERR_BAD_SHAPE;
    if (D == 0) return XTC_OK;
    if (T > kMostExtent || D > kMostExtent || (T > 0 && (lddy > kMostStride || ldx > kMostStride ||
        lddx > kMostStride || (DR && lddr > kMostStride))))
        return XTC_ERR_TOO_LARGE;
    if (T > 0 && (lddy < D || ldx < D || lddx < D || (DR && lddr < D))) return XTC_ERR_BAD_LEADING_DIM;
    if (!DW || (T > 0 && (!DY || !X || !W || !rstd || !DX || !workspace))) return XTC_ERR_NULL_POINTER;
    const int64_t e = size_of(dtype);
    if (!aligned_to(DY, e) || !aligned_to(X, e) || !aligned_to(DR, e) || !aligned_to(DX, e) ||
        !aligned_to(W, size_of(w_dtype)) || !aligned_to(rstd, 4) || !aligned_to(DW, 4) || !aligned_to(workspace, 16))
        return XTC_ERR_MISALIGNED;
    if (workspace_bytes < xtc_rmsnorm_backward_workspace(T, D)) return XTC_ERR_BAD_SHAPE;
    NormBackwardArgs a;
    a.T = T; a.D = (int)D;
    a.DY = DY; a.lddy = lddy; a.X = X; a.ldx = ldx;
    a.W = W; a.w_f32 = w_dtype == XTC_F32; a.rstd = rstd;
    a.DR = DR; a.lddr = lddr; a.DX = DX; a.lddx = lddx;
    a.DW = DW; a.partial = static_cast<float *>(workspace);
    return launch_rmsnorm_backward(a, dtype, static_cast<hipStream_t>(stream));
}

xtc_status xtc_quantize_fp8(int64_t M, int64_t K, const void *X, int64_t ldx, int64_t block_rows, void *Q, int64_t ldq,
                            float *S, int64_t lds, xtc_dtype dtype, void *stream) {
    if (!known(dtype)) return XTC_ERR_BAD_DTYPE;
    if (M < 0 || K < 0 || (block_rows != 1 && block_rows != kScaleBlock)) return XTC_ERR_BAD_SHAPE;
    if (M == 0 || K == 0) return XTC_OK;
    if (M > kMostExtent || K > kMostExtent || ldx > kMostStride || ldq > kMostStride || lds > kMostStride)
        return XTC_ERR_TOO_LARGE;
    if (ldx < K || ldq < K || lds < scale_blocks(K)) return XTC_ERR_BAD_LEADING_DIM;
    if (!X || !Q || !S) return XTC_ERR_NULL_POINTER;
    if (!aligned_to(X, size_of(dtype)) || !aligned_to(S, 4)) return XTC_ERR_MISALIGNED;
    QuantArgs a;
    a.M = M; a.K = K; a.X = X; a.ldx = ldx; a.block_rows = (int)block_rows;
    a.Q = static_cast<uint8_t *>(Q); a.ldq = ldq; a.S = S; a.lds = lds;
    return launch_quantize(a, dtype, static_cast<hipStream_t>(stream));
}

}  // extern "C"

namespace {

// The checks that all products share; `b_rows` x `b_cols` is B of one group.
xtc_status check_product(const GroupedArgs &a, int64_t N, int64_t K, int64_t G, int64_t b_cols, int64_t b_rows,
                         int64_t c_cols, xtc_dtype out_dtype, int64_t elt) {
    if (a.T > kMostExtent || N > kMostExtent || K > kMostExtent || G > kMostExtent || a.lda > kMostStride ||
        a.ldb > kMostStride || a.ldc > kMostStride || (G > 1 && a.stride_b > kMostStride << 20))
        return XTC_ERR_TOO_LARGE;
    if (a.lda < least(K) || a.ldb < least(b_cols) || a.ldc < least(c_cols)) return XTC_ERR_BAD_LEADING_DIM;
    if (G > 1 && b_rows > 0 && a.stride_b < (b_rows - 1) * a.ldb + b_cols) return XTC_ERR_BAD_LEADING_DIM;
    if (!aligned_to(a.A, elt) || !aligned_to(a.B, elt) || !aligned_to(a.C, size_of(out_dtype)) ||
        !aligned_to(a.SA, 4) || !aligned_to(a.SB, 4) || !aligned_to(a.ends, 4))
        return XTC_ERR_MISALIGNED;
    return XTC_OK;
}

xtc_status fp8_product(int64_t G, int64_t T, int64_t N, int64_t K, const void *A, int64_t lda, const float *SA,
                       int64_t ldsa, const void *B, int64_t ldb, int64_t stride_b, const float *SB, int64_t ldsb,
                       int64_t stride_sb, const int32_t *ends, void *C, int64_t ldc, xtc_dtype out_dtype, int32_t relu,
                       void *stream) {
    if (!known(out_dtype)) return XTC_ERR_BAD_DTYPE;
    if (T < 0 || N < 0 || K < 0 || G < 1) return XTC_ERR_BAD_SHAPE;
    GroupedArgs a = {};
    a.T = T; a.N = (int)N; a.K = (int)K;
    a.A = A; a.lda = lda; a.SA = SA; a.ldsa = ldsa;
    a.B = B; a.ldb = ldb; a.stride_b = stride_b; a.SB = SB; a.ldsb = ldsb; a.stride_sb = stride_sb;
    a.C = C; a.ldc = ldc; a.ends = ends; a.G = (int)G;
    a.out_bf16 = out_dtype == XTC_BF16; a.relu = relu != 0;
    const xtc_status st = check_product(a, N, K, G, K, N, N, out_dtype, 1);
    if (st != XTC_OK) return st;
    const int64_t kb = scale_blocks(K), nb = scale_blocks(N);
    if (ldsa > kMostStride || ldsb > kMostStride || stride_sb > kMostStride << 20) return XTC_ERR_TOO_LARGE;
    if (ldsa < least(kb) || ldsb < least(kb) || (G > 1 && nb > 0 && stride_sb < (nb - 1) * ldsb + kb))
        return XTC_ERR_BAD_LEADING_DIM;
    if (T == 0 || N == 0) return XTC_OK;
    if (!C || (K > 0 && (!A || !B || !SA || !SB))) return XTC_ERR_NULL_POINTER;
    return launch_grouped_fp8(a, static_cast<hipStream_t>(stream));
}

}  // namespace

extern "C" {

xtc_status xtc_matmul_fp8(int64_t M, int64_t N, int64_t K, const void *A, int64_t lda, const float *SA, int64_t ldsa,
                          const void *B, int64_t ldb, const float *SB, int64_t ldsb, void *C, int64_t ldc,
                          xtc_dtype out_dtype, int32_t relu, void *stream) {
    return fp8_product(1, M, N, K, A, lda, SA, ldsa, B, ldb, 0, SB, ldsb, 0, nullptr, C, ldc, out_dtype, relu, stream);
}

xtc_status xtc_matmul_grouped_fp8(int64_t G, int64_t T, int64_t N, int64_t K, const void *A, int64_t lda,
                                  const float *SA, int64_t ldsa, const void *B, int64_t ldb, int64_t stride_b,
                                  const float *SB, int64_t ldsb, int64_t stride_sb, const int32_t *ends, void *C,
                                  int64_t ldc, xtc_dtype out_dtype, int32_t relu, void *stream) {
    if (!ends && T > 0 && N > 0) return XTC_ERR_NULL_POINTER;
    return fp8_product(G, T, N, K, A, lda, SA, ldsa, B, ldb, stride_b, SB, ldsb, stride_sb, ends, C, ldc, out_dtype,
                       relu, stream);
}

xtc_status xtc_matmul_grouped(int64_t G, int64_t T, int64_t N, int64_t K, const void *A, int64_t lda, const void *B,
                              int64_t ldb, int64_t stride_b, int32_t transpose_b, const int32_t *ends, void *C,
                              int64_t ldc, xtc_dtype dtype, xtc_dtype out_dtype, int32_t relu, void *stream) {
    if (dtype != XTC_BF16 || !known(out_dtype)) return XTC_ERR_BAD_DTYPE;
    if (T < 0 || N < 0 || K < 0 || G < 1) return XTC_ERR_BAD_SHAPE;
    GroupedArgs a = {};
    a.T = T; a.N = (int)N; a.K = (int)K;
    a.A = A; a.lda = lda; a.B = B; a.ldb = ldb; a.stride_b = stride_b;
    a.C = C; a.ldc = ldc; a.ends = ends; a.G = (int)G;
    a.out_bf16 = out_dtype == XTC_BF16; a.relu = relu != 0;
    const xtc_status st =
        check_product(a, N, K, G, transpose_b ? K : N, transpose_b ? N : K, N, out_dtype, 2);
    if (st != XTC_OK) return st;
    if (T == 0 || N == 0) return XTC_OK;
    if (!C || !ends || (K > 0 && (!A || !B))) return XTC_ERR_NULL_POINTER;
    return launch_grouped_bf16(a, transpose_b != 0, static_cast<hipStream_t>(stream));
}

xtc_status xtc_matmul_grouped_wgrad(int64_t G, int64_t T, int64_t N, int64_t K, const void *A, int64_t lda,
                                    const void *DY, int64_t lddy, const int32_t *ends, void *DB, int64_t lddb,
                                    int64_t stride_db, xtc_dtype dtype, xtc_dtype out_dtype, void *stream) {
    if (dtype != XTC_BF16 || !known(out_dtype)) return XTC_ERR_BAD_DTYPE;
    if (T < 0 || N < 0 || K < 0 || G < 1) return XTC_ERR_BAD_SHAPE;
    GroupedArgs a = {};
    a.T = T; a.N = (int)N; a.K = (int)K;
    a.A = A; a.lda = lda; a.B = DY; a.ldb = lddy;
    a.C = DB; a.ldc = lddb; a.stride_c = stride_db; a.ends = ends; a.G = (int)G;
    a.out_bf16 = out_dtype == XTC_BF16;
    const xtc_status st = check_product(a, N, K, 1, N, T, N, out_dtype, 2);
    if (st != XTC_OK) return st;
    if (G > kMostExtent || stride_db > kMostStride << 20) return XTC_ERR_TOO_LARGE;
    if (G > 1 && K > 0 && stride_db < (K - 1) * lddb + N) return XTC_ERR_BAD_LEADING_DIM;
    if (N == 0 || K == 0) return XTC_OK;
    if (!DB || !ends || (T > 0 && (!A || !DY))) return XTC_ERR_NULL_POINTER;
    return launch_grouped_wgrad(a, static_cast<hipStream_t>(stream));
}

// Not part of the ABI: the kernel of a product of contiguous, 16-byte aligned
// operands (`grouped`: with ends), as grouped_kernel() numbers them, so that the tests
// can see that their sizes reach every one.  Pure host function.
int32_t xtc_test_product_kernel(int32_t kind, int32_t grouped, int64_t G, int64_t T, int64_t N, int64_t K,
                                int32_t out_bf16, int32_t *kernels) {
    static const int32_t ends = 0;
    GroupedArgs a = {};
    a.T = T; a.N = (int)N; a.K = (int)K;
    a.lda = K; a.ldb = kind == 1 || kind == 3 ? N : K;
    a.stride_b = kind == 3 ? 0 : N * K;
    a.ldsa = a.ldsb = scale_blocks(K); a.stride_sb = scale_blocks(N) * a.ldsb;
    a.ldc = N; a.stride_c = N * K;
    a.ends = grouped ? &ends : nullptr; a.G = (int)G;
    a.out_bf16 = out_bf16;
    return grouped_kernel(a, kind, kernels);
}

}  // extern "C"

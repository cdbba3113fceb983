"""Refusals of the norm, 8-bit and grouped operators, on the CPU: every invalid
call returns its status before the device is touched (the pointers are NULL or
dummies), and the conveniences over tensors raise."""
import pytest

import paper_2512_16512_amd as x

BAD = 0x1000   # a dummy non-NULL pointer on every alignment boundary
BIG = 1 << 40


def call(fn, good, **change):
    assert set(change) <= set(good), change
    return fn(**{**good, **change})


NORM = dict(T=4, D=200, X=BAD, ldx=200, R=BAD, ldr=200, W=BAD, eps=1e-6, Y=BAD, ldy=200, S=BAD, lds=2, H=BAD, ldh=200,
            rstd=BAD, dtype=1, w_dtype=1, out_dtype=2)


@pytest.mark.parametrize("change,status", [
    (dict(dtype=2), 4), (dict(dtype=7), 4), (dict(w_dtype=2), 4), (dict(out_dtype=0), 4), (dict(dtype=0, w_dtype=1), 4),
    (dict(T=-1), 2), (dict(D=-1), 2), (dict(eps=-1.0), 2), (dict(eps=float("nan")), 2),
    (dict(ldx=199), 3), (dict(ldr=199), 3), (dict(ldy=199), 3), (dict(ldh=199), 3), (dict(lds=1), 3),
    (dict(X=0), 1), (dict(W=0), 1), (dict(Y=0), 1), (dict(S=0), 1), (dict(R=0, ldr=0), 1),
    (dict(X=BAD + 1), 9), (dict(R=BAD + 1), 9), (dict(W=BAD + 1), 9), (dict(w_dtype=0, W=BAD + 2), 9),
    (dict(S=BAD + 2), 9), (dict(H=BAD + 1), 9), (dict(rstd=BAD + 2), 9), (dict(out_dtype=1, Y=BAD + 1), 9),
    (dict(T=BIG), 7), (dict(D=BIG, ldx=BIG, ldr=BIG, ldy=BIG, ldh=BIG), 7), (dict(ldx=BIG), 7),
    (dict(T=0, X=0), 0), (dict(D=0, Y=0), 0),
])
def test_rmsnorm_refuses(change, status):
    assert call(x.xtc_rmsnorm, NORM, **change) == status


BACK = dict(T=4, D=200, DY=BAD, lddy=200, X=BAD, ldx=200, W=BAD, rstd=BAD, DR=BAD, lddr=200, DX=BAD, lddx=200, DW=BAD,
            workspace=BAD, workspace_bytes=1 << 20, dtype=0, w_dtype=0)


@pytest.mark.parametrize("change,status", [
    (dict(dtype=2), 4), (dict(w_dtype=1), 4), (dict(T=-1), 2), (dict(D=-1), 2), (dict(workspace_bytes=x.xtc_rmsnorm_backward_workspace(4, 200) - 1), 2),
    (dict(lddy=199), 3), (dict(ldx=199), 3), (dict(lddr=199), 3), (dict(lddx=199), 3),
    (dict(DY=0), 1), (dict(X=0), 1), (dict(W=0), 1), (dict(rstd=0), 1), (dict(DX=0), 1), (dict(DW=0), 1),
    (dict(workspace=0), 1), (dict(DX=BAD + 2), 9), (dict(workspace=BAD + 4), 9), (dict(T=BIG), 7), (dict(lddx=BIG), 7),
    (dict(D=0), 0),
])
def test_rmsnorm_backward_refuses(change, status):
    assert call(x.xtc_rmsnorm_backward, BACK, **change) == status


def test_rmsnorm_backward_workspace():
    assert x.xtc_rmsnorm_backward_workspace(-1, 4) == -1 and x.xtc_rmsnorm_backward_workspace(4, BIG) == -1
    assert x.xtc_rmsnorm_backward_workspace(0, 100) == 0 or x.xtc_rmsnorm_backward_workspace(0, 100) > 0
    assert x.xtc_rmsnorm_backward_workspace(4, 200) >= 4 * 200


@pytest.mark.parametrize("T,D,slabs", [(0, 100, 0), (4, 200, 1), (5, 200, 2), (8191, 500, 1024), (8191, 1000, 768),
                                       (8191, 2048, 1024), (8191, 4096, 768), (8191, 8192, 256), (300, 9000, 300),
                                       (8191, 9000, 512)])
def test_rmsnorm_backward_workspace_holds_a_row_of_sums_for_each_workgroup(T, D, slabs):
    assert x.xtc_rmsnorm_backward_workspace(T, D) == 4 * slabs * D


QUANT = dict(M=4, K=200, X=BAD, ldx=200, block_rows=1, Q=BAD, ldq=200, S=BAD, lds=2, dtype=0)


@pytest.mark.parametrize("change,status", [
    (dict(dtype=2), 4), (dict(M=-1), 2), (dict(K=-1), 2), (dict(block_rows=2), 2), (dict(block_rows=0), 2),
    (dict(ldx=199), 3), (dict(ldq=199), 3), (dict(lds=1), 3), (dict(X=0), 1), (dict(Q=0), 1), (dict(S=0), 1),
    (dict(X=BAD + 2), 9), (dict(S=BAD + 1), 9), (dict(M=BIG), 7), (dict(ldq=BIG), 7), (dict(M=0, X=0), 0),
])
def test_quantize_refuses(change, status):
    assert call(x.xtc_quantize_fp8, QUANT, **change) == status


FP8 = dict(M=4, N=130, K=200, A=BAD, lda=200, SA=BAD, ldsa=2, B=BAD, ldb=200, SB=BAD, ldsb=2, C=BAD, ldc=130, out_dtype=0)


@pytest.mark.parametrize("change,status", [
    (dict(out_dtype=2), 4), (dict(M=-1), 2), (dict(N=-1), 2), (dict(K=-1), 2),
    (dict(lda=199), 3), (dict(ldb=199), 3), (dict(ldc=129), 3), (dict(ldsa=1), 3), (dict(ldsb=1), 3),
    (dict(A=0), 1), (dict(B=0), 1), (dict(SA=0), 1), (dict(SB=0), 1), (dict(C=0), 1),
    (dict(SA=BAD + 2), 9), (dict(SB=BAD + 2), 9), (dict(C=BAD + 2), 9), (dict(out_dtype=1, C=BAD + 1), 9),
    (dict(M=BIG), 7), (dict(N=BIG), 7), (dict(K=BIG), 7), (dict(lda=BIG), 7), (dict(ldsa=BIG), 7),
    (dict(M=0x7FFFFF00, N=0x7FFFFF00, ldc=1 << 30, A=0), 3), (dict(M=1 << 30, N=1 << 30, ldc=1 << 30), 7),
    (dict(M=0, A=0), 0), (dict(N=0, B=0, C=0), 0),
])
def test_matmul_fp8_refuses(change, status):
    assert call(x.xtc_matmul_fp8, FP8, **change) == status


GROUPED = dict(G=3, T=4, N=130, K=200, A=BAD, lda=200, B=BAD, ldb=130, stride_b=26000, transpose_b=0, ends=BAD, C=BAD,
               ldc=130, dtype=1, out_dtype=0)


@pytest.mark.parametrize("change,status", [
    (dict(dtype=0), 4), (dict(dtype=2), 4), (dict(out_dtype=2), 4), (dict(G=0), 2), (dict(T=-1), 2), (dict(N=-1), 2),
    (dict(K=-1), 2), (dict(lda=199), 3), (dict(ldb=129), 3), (dict(ldb=199, transpose_b=1), 3), (dict(ldc=129), 3),
    (dict(stride_b=25999), 3), (dict(stride_b=0), 3), (dict(A=0), 1), (dict(B=0), 1), (dict(C=0), 1), (dict(ends=0), 1),
    (dict(A=BAD + 1), 9), (dict(ends=BAD + 2), 9), (dict(G=BIG), 7), (dict(T=BIG), 7), (dict(ldb=BIG), 7),
    (dict(T=0, A=0), 0), (dict(N=0, ldb=1), 0),
])
def test_matmul_grouped_refuses(change, status):
    assert call(x.xtc_matmul_grouped, GROUPED, **change) == status


WGRAD = dict(G=3, T=4, N=130, K=200, A=BAD, lda=200, DY=BAD, lddy=130, ends=BAD, DB=BAD, lddb=130, stride_db=26000,
             dtype=1, out_dtype=0)


@pytest.mark.parametrize("change,status", [
    (dict(dtype=0), 4), (dict(out_dtype=2), 4), (dict(G=0), 2), (dict(T=-1), 2), (dict(lda=199), 3),
    (dict(lddy=129), 3), (dict(lddb=129), 3), (dict(stride_db=25999), 3), (dict(A=0), 1), (dict(DY=0), 1),
    (dict(DB=0), 1), (dict(ends=0), 1), (dict(DY=BAD + 1), 9), (dict(DB=BAD + 2), 9), (dict(G=BIG), 7),
    (dict(N=0, lddy=1, lddb=1), 0), (dict(K=0, lda=1, DB=0), 0),
])
def test_matmul_grouped_wgrad_refuses(change, status):
    assert call(x.xtc_matmul_grouped_wgrad, WGRAD, **change) == status


GROUPED_FP8 = dict(G=3, T=4, N=130, K=200, A=BAD, lda=200, SA=BAD, ldsa=2, B=BAD, ldb=200, stride_b=26000, SB=BAD, ldsb=2,
                   stride_sb=4, ends=BAD, C=BAD, ldc=130, out_dtype=1)


@pytest.mark.parametrize("change,status", [
    (dict(out_dtype=2), 4), (dict(G=0), 2), (dict(G=-3), 2), (dict(stride_b=25999), 3), (dict(stride_sb=3), 3),
    (dict(ldsb=1), 3), (dict(ends=0), 1), (dict(SB=0), 1), (dict(SB=BAD + 2), 9), (dict(stride_sb=1 << 60), 7),
    (dict(T=0, ends=0, A=0), 0),
])
def test_matmul_grouped_fp8_refuses(change, status):
    assert call(x.xtc_matmul_grouped_fp8, GROUPED_FP8, **change) == status


# ------------------------------------------------ the conveniences' own checks


torch = pytest.importorskip("torch")


def t(*shape, dtype=torch.bfloat16):
    return torch.zeros(*shape).to(dtype)


E4M3 = torch.float8_e4m3fn


@pytest.mark.parametrize("fn,args,error,match", [
    (x.rmsnorm, (t(4, 8, dtype=torch.float16), t(8)), TypeError, "x must be float32 or bfloat16"),
    (x.rmsnorm, (t(4, 8), t(8)), ValueError, "CUDA"),
    (x.rmsnorm, (t(8, 4).t(), t(8)), ValueError, "unit stride"),
    (x.rmsnorm, (t(8), t(8)), ValueError, "2-D"),
    (x.rmsnorm_backward, (t(4, 8), t(4, 8, dtype=E4M3), t(8), t(4)), TypeError, "x must be"),
    (x.quantize_fp8, (t(4, 8, dtype=E4M3),), TypeError, "x must be"),
    (x.quantize_fp8, (t(4, 8),), ValueError, "CUDA"),
    (x.matmul_fp8, (t(4, 8), t(4, 1), t(4, 8), t(1, 1)), TypeError, "a must be float8_e4m3fn"),
    (x.matmul_fp8, (t(4, 8, dtype=E4M3), t(4, 1), t(4, 8, dtype=E4M3), t(1, 1)), ValueError, "CUDA"),
    (x.matmul_grouped, (t(4, 8, dtype=torch.float32), t(2, 8, 4), t(2)), TypeError, "a must be bfloat16"),
    (x.matmul_grouped, (t(4, 8), t(2, 8, 4), t(2)), ValueError, "CUDA"),
    (x.matmul_grouped_wgrad, (t(4, 8), t(4, 4), t(2)), ValueError, "CUDA"),
    (x.matmul_grouped_fp8, (t(4, 8), t(4, 1), t(2, 4, 8), t(2, 1, 1), t(2)), TypeError, "a must be float8_e4m3fn"),
])
def test_conveniences_refuse(fn, args, error, match):
    with pytest.raises(error, match=match):
        fn(*args)


def test_the_native_entries_leave_other_tensors_to_python():
    a, i = t(4, 8), torch.zeros(2, dtype=torch.int32)
    q = t(4, 8, dtype=E4M3)
    for name, args in (("rmsnorm", (a, t(8), None, 1e-6, False)), ("rmsnorm_backward", (a, a, t(8), t(4), None)),
                       ("quantize_fp8", (a, 1)), ("matmul_fp8", (q, t(4, 1), q, t(1, 1), None, False, None)),
                       ("matmul_grouped", (a, t(2, 8, 4), i, False, None, False, None)),
                       ("matmul_grouped_wgrad", (a, a, i, None, None)),
                       ("matmul_grouped_fp8", (q, t(4, 1), t(2, 4, 8, dtype=E4M3), t(2, 1, 1), i, None, False, None))):
        fast = getattr(x._fast, name)
        assert fast(*args) is None and fast() is None and fast(*([None] * len(args))) is None


@pytest.mark.gpu
def test_conveniences_refuse_on_the_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU visible")

    def c(*shape, dtype=torch.bfloat16):
        return t(*shape, dtype=dtype).cuda()

    f32, i32 = torch.float32, torch.int32
    cases = [
        (lambda: x.rmsnorm(c(4, 8), c(9)), ValueError, "weight must be a contiguous vector of 8"),
        (lambda: x.rmsnorm(c(4, 8, dtype=f32), c(8)), TypeError, "weight must be float32"),
        (lambda: x.rmsnorm(c(4, 8), c(8), c(4, 9)), ValueError, "residual must be"),
        (lambda: x.rmsnorm(c(4, 8), c(8), c(4, 8, dtype=f32)), TypeError, "residual must be bfloat16"),
        (lambda: x.rmsnorm(c(4, 8), t(8)), ValueError, "weight must be on"),
        (lambda: x.rmsnorm(c(4, 8), c(8), eps=-1.0), x.XtcError, "inconsistent|extent|shape"),
        (lambda: x.rmsnorm(c(1, 8).expand(4, 8), c(8)), x.XtcError, "leading|stride"),
        (lambda: x.rmsnorm_backward(c(3, 8), c(4, 8), c(8), c(4, dtype=f32)), ValueError, "dy must be"),
        (lambda: x.rmsnorm_backward(c(4, 8), c(4, 8), c(8), c(4)), TypeError, "rstd must be float32"),
        (lambda: x.quantize_fp8(c(4, 8), block_rows=64), ValueError, "block_rows"),
        (lambda: x.matmul_fp8(c(4, 8, dtype=E4M3), c(4, 1, dtype=f32), c(4, 9, dtype=E4M3), c(1, 1, dtype=f32)),
         ValueError, "inner dimensions differ"),
        (lambda: x.matmul_fp8(c(4, 8, dtype=E4M3), c(4, 2, dtype=f32), c(4, 8, dtype=E4M3), c(1, 1, dtype=f32)),
         ValueError, "a_scale must be"),
        (lambda: x.matmul_fp8(c(4, 8, dtype=E4M3), c(4, 1, dtype=f32), c(4, 8, dtype=E4M3), c(1, 1, dtype=f32),
                              dtype=torch.float16), TypeError, "dtype must be"),
        (lambda: x.matmul_fp8(c(4, 8, dtype=E4M3), c(4, 1, dtype=f32), c(4, 8, dtype=E4M3), c(1, 1, dtype=f32),
                              out=c(4, 5, dtype=f32)), ValueError, "out must be"),
        (lambda: x.matmul_grouped(c(4, 8), c(8, 4), c(2, dtype=i32)), ValueError, "3-D"),
        (lambda: x.matmul_grouped(c(4, 8), c(2, 7, 4), c(2, dtype=i32)), ValueError, "b must be"),
        (lambda: x.matmul_grouped(c(4, 8), c(2, 8, 4), c(3, dtype=i32)), ValueError, "ends must be"),
        (lambda: x.matmul_grouped(c(4, 8), c(2, 8, 4), c(2, dtype=torch.int64)), TypeError, "ends must be int32"),
        (lambda: x.matmul_grouped(c(4, 8), c(1, 8, 4).expand(2, 8, 4), c(2, dtype=i32)), x.XtcError, "leading|stride"),
        (lambda: x.matmul_grouped(c(4, 8), c(0, 8, 4), c(0, dtype=i32)), x.XtcError, "extent|shape"),
        (lambda: x.matmul_grouped_wgrad(c(4, 8), c(5, 4), c(2, dtype=i32)), ValueError, "rows"),
        (lambda: x.matmul_grouped_fp8(c(4, 8, dtype=E4M3), c(4, 1, dtype=f32), c(2, 4, 8, dtype=E4M3),
                                      c(2, 2, 1, dtype=f32), c(2, dtype=i32)), ValueError, "b_scale must be"),
    ]
    for make, error, match in cases:
        with pytest.raises(error, match=match):
            make()

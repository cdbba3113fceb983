"""Refusals of the layer norm, linear, routing and combining operators, on the CPU:
every invalid call returns its status before the device is touched (the pointers are
NULL or dummies), and the conveniences over tensors raise."""
import pytest

import paper_2512_16512_amd as x
from test_operators_abi import BAD, BIG, E4M3, call, t

torch = pytest.importorskip("torch")

NORM = dict(T=4, D=200, X=BAD, ldx=200, R=BAD, ldr=200, W=BAD, B=BAD, eps=1e-6, Y=BAD, ldy=200, S=BAD, lds=2, H=BAD,
            ldh=200, mean=BAD, rstd=BAD, dtype=1, w_dtype=1, out_dtype=2)


@pytest.mark.parametrize("change,status", [
    (dict(dtype=2), 4), (dict(dtype=7), 4), (dict(w_dtype=2), 4), (dict(out_dtype=0), 4), (dict(dtype=0, w_dtype=1), 4),
    (dict(T=-1), 2), (dict(D=-1), 2), (dict(eps=-1.0), 2), (dict(eps=float("nan")), 2),
    (dict(ldx=199), 3), (dict(ldr=199), 3), (dict(ldy=199), 3), (dict(ldh=199), 3), (dict(lds=1), 3),
    (dict(X=0), 1), (dict(W=0), 1), (dict(Y=0), 1), (dict(S=0), 1), (dict(R=0, ldr=0), 1),
    (dict(X=BAD + 1), 9), (dict(R=BAD + 1), 9), (dict(W=BAD + 1), 9), (dict(B=BAD + 1), 9), (dict(w_dtype=0, B=BAD + 2), 9),
    (dict(S=BAD + 2), 9), (dict(H=BAD + 1), 9), (dict(rstd=BAD + 2), 9), (dict(mean=BAD + 2), 9),
    (dict(out_dtype=1, Y=BAD + 1), 9), (dict(T=BIG), 7), (dict(D=BIG, ldx=BIG, ldr=BIG, ldy=BIG, ldh=BIG), 7),
    (dict(ldx=BIG), 7), (dict(T=0, X=0), 0), (dict(D=0, Y=0), 0),
])
def test_layernorm_refuses(change, status):
    assert call(x.xtc_layernorm, NORM, **change) == status


BACK = dict(T=4, D=200, DY=BAD, lddy=200, X=BAD, ldx=200, W=BAD, mean=BAD, rstd=BAD, DR=BAD, lddr=200, DX=BAD, lddx=200,
            DW=BAD, DB=BAD, workspace=BAD, workspace_bytes=1 << 20, dtype=0, w_dtype=0)


@pytest.mark.parametrize("change,status", [
    (dict(dtype=2), 4), (dict(w_dtype=1), 4), (dict(T=-1), 2), (dict(D=-1), 2),
    (dict(workspace_bytes=x.xtc_layernorm_backward_workspace(4, 200) - 1), 2),
    (dict(lddy=199), 3), (dict(ldx=199), 3), (dict(lddr=199), 3), (dict(lddx=199), 3),
    (dict(DY=0), 1), (dict(X=0), 1), (dict(W=0), 1), (dict(mean=0), 1), (dict(rstd=0), 1), (dict(DX=0), 1), (dict(DW=0), 1),
    (dict(DB=0), 1), (dict(workspace=0), 1), (dict(DX=BAD + 2), 9), (dict(mean=BAD + 2), 9), (dict(DB=BAD + 2), 9),
    (dict(workspace=BAD + 4), 9), (dict(T=BIG), 7), (dict(lddx=BIG), 7), (dict(D=0), 0),
])
def test_layernorm_backward_refuses(change, status):
    assert call(x.xtc_layernorm_backward, BACK, **change) == status


def test_layernorm_backward_workspace():
    assert x.xtc_layernorm_backward_workspace(-1, 4) == -1 and x.xtc_layernorm_backward_workspace(4, BIG) == -1
    assert x.xtc_layernorm_backward_workspace(0, 100) >= 0
    assert x.xtc_layernorm_backward_workspace(4, 200) >= 8 * 200


LINEAR = dict(T=4, N=130, K=200, A=BAD, lda=200, B=BAD, ldb=130, transpose_b=0, bias=BAD, bias_dtype=0, R=BAD, ldr=130,
              r_dtype=1, activation=2, C=BAD, ldc=130, Z=BAD, ldz=130, workspace=BAD, workspace_bytes=1 << 30, dtype=1,
              out_dtype=1)


@pytest.mark.parametrize("change,status", [
    (dict(dtype=0), 4), (dict(dtype=2), 4), (dict(out_dtype=2), 4), (dict(bias_dtype=2), 4), (dict(r_dtype=2), 4),
    (dict(T=-1), 2), (dict(N=-1), 2), (dict(K=-1), 2), (dict(activation=-1), 2), (dict(activation=5), 2),
    (dict(lda=199), 3), (dict(ldb=129), 3), (dict(ldb=199, transpose_b=1), 3), (dict(ldc=129), 3), (dict(ldr=129), 3),
    (dict(ldz=129), 3), (dict(A=0), 1), (dict(B=0), 1), (dict(C=0), 1),
    (dict(A=BAD + 1), 9), (dict(B=BAD + 1), 9), (dict(bias=BAD + 2), 9), (dict(R=BAD + 1), 9), (dict(C=BAD + 1), 9),
    (dict(Z=BAD + 1), 9), (dict(out_dtype=0, C=BAD + 2), 9), (dict(workspace=BAD + 8), 9),
    (dict(T=BIG), 7), (dict(N=BIG), 7), (dict(K=BIG), 7), (dict(lda=BIG), 7), (dict(ldr=BIG), 7), (dict(ldz=BIG), 7),
    (dict(T=1 << 30, N=1 << 30, ldb=1 << 30, ldc=1 << 30, ldr=1 << 30, ldz=1 << 30, workspace_bytes=1 << 62), 7),
    (dict(T=0, A=0), 0), (dict(N=0, B=0, C=0), 0), (dict(N=0, ldb=1, ldc=1, ldr=1, ldz=1), 0),
])
def test_linear_refuses(change, status):
    assert call(x.xtc_linear, LINEAR, **change) == status


def test_linear_workspaces():
    assert x.xtc_linear_workspace(-1, 4, 4, BAD, 8, BAD, 8, 0) == -1 and x.xtc_linear_workspace(4, 4, BIG, BAD, 8, BAD, 8, 0) == -1
    assert x.xtc_linear_wgrad_workspace(4, -1, 4, BAD, 8, BAD, 8) == -1 and x.xtc_activation_backward_workspace(BIG, 4) == -1
    assert x.xtc_linear_workspace(0, 4, 4, BAD, 8, BAD, 8, 0) == 0 and x.xtc_linear_wgrad_workspace(4, 0, 4, BAD, 8, BAD, 8) == 0
    # a reduction long enough that its parts go to several workgroups, each part's sums a whole result
    need = x.xtc_linear_wgrad_workspace(16384, 256, 256, BAD, 256, BAD, 256)
    assert need > 0 and need % (4 * 256 * 256) == 0
    assert call(x.xtc_linear_wgrad, WGRAD, T=16384, N=256, K=256, lda=256, lddy=256, lddb=256, workspace_bytes=need - 1) == 2
    assert call(x.xtc_linear_wgrad, WGRAD, T=16384, N=256, K=256, lda=256, lddy=256, lddb=256, workspace_bytes=need,
                workspace=0) == 1
    assert x.xtc_activation_backward_workspace(4, 200) >= 4 * 200 and x.xtc_activation_backward_workspace(0, 200) >= 4 * 200


WGRAD = dict(T=4, N=130, K=200, A=BAD, lda=200, DY=BAD, lddy=130, DB=BAD, lddb=130, workspace=BAD,
             workspace_bytes=1 << 30, dtype=1, out_dtype=0)


@pytest.mark.parametrize("change,status", [
    (dict(dtype=0), 4), (dict(out_dtype=2), 4), (dict(T=-1), 2), (dict(N=-1), 2), (dict(K=-1), 2), (dict(lda=199), 3),
    (dict(lddy=129), 3), (dict(lddb=129), 3), (dict(A=0), 1), (dict(DY=0), 1), (dict(DB=0), 1), (dict(DY=BAD + 1), 9),
    (dict(DB=BAD + 2), 9), (dict(workspace=BAD + 4), 9), (dict(T=BIG), 7), (dict(lddb=BIG), 7),
    (dict(N=0, lddy=1, lddb=1), 0), (dict(K=0, lda=1, DB=0), 0),
])
def test_linear_wgrad_refuses(change, status):
    assert call(x.xtc_linear_wgrad, WGRAD, **change) == status


SLOPE = dict(T=4, N=130, DY=BAD, lddy=130, dy_dtype=1, Z=BAD, ldz=130, z_dtype=0, activation=3, DZ=BAD, lddz=130, DB=BAD,
             workspace=BAD, workspace_bytes=1 << 30)


@pytest.mark.parametrize("change,status", [
    (dict(dy_dtype=2), 4), (dict(z_dtype=2), 4), (dict(T=-1), 2), (dict(N=-1), 2), (dict(activation=5), 2),
    (dict(activation=-1), 2), (dict(workspace_bytes=x.xtc_activation_backward_workspace(4, 130) - 1), 2),
    (dict(lddy=129), 3), (dict(ldz=129), 3), (dict(lddz=129), 3), (dict(DY=0), 1), (dict(Z=0), 1), (dict(DZ=0), 1),
    (dict(workspace=0), 1), (dict(DY=BAD + 1), 9), (dict(Z=BAD + 2), 9), (dict(DZ=BAD + 1), 9), (dict(DB=BAD + 2), 9),
    (dict(workspace=BAD + 8), 9), (dict(T=BIG), 7), (dict(lddz=BIG), 7), (dict(N=0), 0), (dict(T=0, DB=0), 0),
])
def test_activation_backward_refuses(change, status):
    assert call(x.xtc_activation_backward, SLOPE, **change) == status


ROUTE = dict(T=4, E=20, top=3, scores=BAD, lds=20, mask=0, expert=BAD, p=BAD, row=BAD, token=BAD, counts=BAD, ends=BAD,
             loss=BAD, workspace=BAD, workspace_bytes=1 << 20, dtype=0)


@pytest.mark.parametrize("change,status", [
    (dict(dtype=2), 4), (dict(T=-1), 2), (dict(E=0), 2), (dict(top=0), 2), (dict(top=21), 2), (dict(top=-1), 2),
    (dict(T=4000, workspace_bytes=x.xtc_route_experts_workspace(4000, 20) - 1), 2), (dict(lds=19), 3),
    (dict(E=1025, lds=1025), 7), (dict(E=64, lds=64, top=17), 7), (dict(T=1 << 30), 7), (dict(T=BIG), 7), (dict(lds=BIG), 7),
    (dict(scores=0), 1), (dict(expert=0), 1), (dict(p=0), 1), (dict(row=0), 1), (dict(token=0), 1), (dict(counts=0), 1),
    (dict(ends=0), 1), (dict(loss=0), 1), (dict(T=4000, workspace=0), 1), (dict(scores=BAD + 2), 9), (dict(expert=BAD + 2), 9),
    (dict(p=BAD + 1), 9), (dict(row=BAD + 2), 9), (dict(token=BAD + 2), 9), (dict(counts=BAD + 2), 9), (dict(ends=BAD + 2), 9),
    (dict(loss=BAD + 2), 9), (dict(workspace=BAD + 4), 9),
])
def test_route_experts_refuses(change, status):
    assert call(x.xtc_route_experts, ROUTE, **change) == status


def test_route_experts_workspace():
    assert x.xtc_route_experts_workspace(-1, 4) == -1 and x.xtc_route_experts_workspace(4, 0) == -1
    assert x.xtc_route_experts_workspace(4, 1025) == -1 and x.xtc_route_experts_workspace(BIG, 4) == -1
    assert x.xtc_route_experts_workspace(0, 20) == 0 and x.xtc_route_experts_workspace(4000, 20) >= 8 * 20


ROUTE_BACK = dict(T=4, E=20, top=3, DP=BAD, scores=BAD, lds=20, expert=BAD, p=BAD, counts=BAD, dloss=0.1, DS=BAD, ldds=20,
                  dtype=0, out_dtype=1)


@pytest.mark.parametrize("change,status", [
    (dict(dtype=2), 4), (dict(out_dtype=2), 4), (dict(T=-1), 2), (dict(E=0), 2), (dict(top=0), 2), (dict(top=21), 2),
    (dict(lds=19), 3), (dict(ldds=19), 3), (dict(E=1025, lds=1025, ldds=1025), 7), (dict(E=64, lds=64, ldds=64, top=17), 7),
    (dict(T=BIG), 7), (dict(ldds=BIG), 7), (dict(scores=0), 1), (dict(expert=0), 1), (dict(p=0), 1), (dict(counts=0), 1),
    (dict(DS=0), 1), (dict(DP=BAD + 2), 9), (dict(scores=BAD + 2), 9), (dict(expert=BAD + 1), 9), (dict(DS=BAD + 1), 9),
    (dict(T=0, scores=0, DS=0), 0),
])
def test_route_experts_backward_refuses(change, status):
    assert call(x.xtc_route_experts_backward, ROUTE_BACK, **change) == status


COMBINE = dict(T=4, top=3, D=40, R=12, rows=BAD, ldrows=40, row=BAD, p=BAD, RES=BAD, ldr=40, r_dtype=0, C=BAD, ldc=40,
               dtype=1, out_dtype=1)


@pytest.mark.parametrize("change,status", [
    (dict(dtype=2), 4), (dict(out_dtype=2), 4), (dict(r_dtype=2), 4), (dict(T=-1), 2), (dict(top=-1), 2), (dict(D=-1), 2),
    (dict(R=-1), 2), (dict(ldrows=39), 3), (dict(ldr=39), 3), (dict(ldc=39), 3), (dict(rows=0), 1), (dict(row=0), 1),
    (dict(C=0), 1), (dict(rows=BAD + 1), 9), (dict(row=BAD + 2), 9), (dict(p=BAD + 2), 9), (dict(RES=BAD + 2), 9),
    (dict(C=BAD + 1), 9), (dict(T=BIG), 7), (dict(T=1 << 30), 7), (dict(D=BIG, ldrows=BIG), 7), (dict(R=BIG), 7),
    (dict(ldc=BIG), 7), (dict(T=0, C=0), 0), (dict(D=0, C=0), 0),
])
def test_combine_experts_refuses(change, status):
    assert call(x.xtc_combine_experts, COMBINE, **change) == status


COMBINE_BACK = dict(T=4, top=3, D=40, DOUT=BAD, lddo=40, dout_dtype=0, rows=BAD, ldrows=40, row=BAD, token=BAD, p=BAD,
                    DROWS=BAD, lddr=40, DP=BAD, dtype=1)


@pytest.mark.parametrize("change,status", [
    (dict(dtype=2), 4), (dict(dout_dtype=2), 4), (dict(T=-1), 2), (dict(top=0), 2), (dict(D=-1), 2), (dict(lddo=39), 3),
    (dict(ldrows=39), 3), (dict(lddr=39), 3), (dict(DOUT=0), 1), (dict(rows=0), 1), (dict(row=0), 1), (dict(token=0), 1),
    (dict(p=0), 1), (dict(DROWS=0), 1), (dict(DP=0), 1), (dict(DOUT=BAD + 2), 9), (dict(rows=BAD + 1), 9),
    (dict(row=BAD + 2), 9), (dict(token=BAD + 2), 9), (dict(p=BAD + 2), 9), (dict(DROWS=BAD + 1), 9), (dict(DP=BAD + 2), 9),
    (dict(T=BIG), 7), (dict(T=1 << 30), 7), (dict(lddr=BIG), 7), (dict(T=0, DOUT=0), 0),
])
def test_combine_experts_backward_refuses(change, status):
    assert call(x.xtc_combine_experts_backward, COMBINE_BACK, **change) == status


# ------------------------------------------------ the conveniences' own checks


F32 = torch.float32


@pytest.mark.parametrize("fn,args,error,match", [
    (x.layernorm, (t(4, 8, dtype=torch.float16), t(8)), TypeError, "x must be float32 or bfloat16"),
    (x.layernorm, (t(4, 8), t(8)), ValueError, "CUDA"),
    (x.layernorm, (t(8, 4).t(), t(8)), ValueError, "unit stride"),
    (x.layernorm_backward, (t(4, 8), t(4, 8, dtype=E4M3), t(8), t(4), t(4)), TypeError, "x must be"),
    (x.layernorm_backward, (t(4, 8), t(4, 8), t(8), t(4), t(4)), ValueError, "CUDA"),
    (x.linear, (t(4, 8, dtype=F32), t(8, 4)), TypeError, "a must be bfloat16"),
    (x.linear, (t(4, 8), t(8, 4)), ValueError, "CUDA"),
    (x.linear, (t(4, 8), t(8, 4), None, None, "tanh"), ValueError, "activation must be"),
    (x.linear_wgrad, (t(4, 8), t(4, 4)), ValueError, "CUDA"),
    (x.activation_backward, (t(4, 8), t(4, 8), "swish"), ValueError, "activation must be"),
    (x.activation_backward, (t(4, 8, dtype=E4M3), t(4, 8), "relu"), TypeError, "dy must be"),
    (x.route_experts, (t(4, 8, dtype=torch.float16), 2), TypeError, "scores must be"),
    (x.route_experts, (t(4, 8), 2), ValueError, "CUDA"),
    (x.route_experts_backward, (None, t(4, 8), t(4, 2), t(4, 2), t(8)), ValueError, "CUDA"),
    (x.combine_experts, (t(4, 8, dtype=E4M3), t(4, 2)), TypeError, "rows must be"),
    (x.combine_experts, (t(8, 8), t(4, 2)), ValueError, "CUDA"),
    (x.combine_experts_backward, (t(4, 8), t(8, 8), t(4, 2), t(8), t(4, 2)), ValueError, "CUDA"),
])
def test_conveniences_refuse(fn, args, error, match):
    with pytest.raises(error, match=match):
        fn(*args)


def test_the_native_entries_leave_other_tensors_to_python():
    a, v, i = t(4, 8), t(4, dtype=F32), torch.zeros(4, 2, dtype=torch.int32)
    for name, args in (("layernorm", (a, t(8), t(8), None, 1e-6, False)), ("layernorm_backward", (a, a, t(8), v, v, None)),
                       ("linear", (a, t(8, 4), None, None, 0, False, False, None, None)),
                       ("linear_wgrad", (a, a, None, None)), ("activation_backward", (a, a, 1)),
                       ("route_experts", (a, 2, None)), ("route_experts_backward", (None, a, i, v, i, 0.0, None)),
                       ("combine_experts", (a, i, None, None, None)), ("combine_experts_backward", (a, a, i, i, v))):
        fast = getattr(x._fast, name)
        assert fast(*args) is None and fast() is None and fast(*([None] * len(args))) is None

"""The layer norm and the linear layer with their gradients against their
definitions in 64 bits.

Tolerances.  u = 2^-24 is half a unit in the last place of fp32.  A sum of n fp32
terms in any order is within n u of the sum of their magnitudes; those along a
row are taken by threads of at most 64 terms each, or a 256th of a longer row's, and
joined by halves: 64 + n / 256 stands for n there.  The matrix cores may truncate where
they add, so products count 2u a term.  Rounding to bf16 is within 2^-8 of the value,
to e4m3 within 2^-4 of it, and within 2^-10 near zero."""
import math

import pytest

from _helpers import say
from test_operators import BF16, U, as_type, check_e4m3, dev, host, normal, within

torch = pytest.importorskip("torch")
x = pytest.importorskip("paper_2512_16512_amd")


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU visible")


pytestmark = pytest.mark.gpu

SIZES = [(1, 1), (3, 7), (2, 127), (5, 128), (4, 129), (1, 4096), (33, 512), (7, 1021), (3, 2050), (6, 1501), (2, 8192),
         (1, 8200), (2, 20001), (1, 40000)]


def depth(n):
    return min(n, 64 + n // 256)


# ------------------------------------------------------------- layer norm


def norm_case(T, D, dtype, residual, seed):
    xs = as_type((normal(seed, T, D) + 2 * normal(seed + 4, 1, D)) * torch.exp(normal(seed + 1, D)), dtype)
    w = as_type(1 + 0.2 * normal(seed + 2, D), dtype)
    b = as_type(0.5 * normal(seed + 5, D), dtype)
    r = as_type(3 * normal(seed + 3, T, D), dtype) if residual else None
    return xs, w, b, r


def norm_reference(xs, w, b, r, eps):
    """h, mean, rstd and y in 64 bits, and how far the kernel's mean, rstd (relative) and unrounded y may be off."""
    D = xs.shape[1]
    h = xs.double() + (r.double() if r is not None else 0)
    mean = h.mean(1)
    d = h - mean[:, None]
    var = d.square().mean(1)
    rstd = 1 / torch.sqrt(var + eps)
    bias = b.double() if b is not None else torch.zeros(D, dtype=torch.float64)
    y = w.double() * d * rstd[:, None] + bias
    e_mean = (depth(D) + 4) * U * h.abs().mean(1)
    e_d = U * h.abs() + e_mean[:, None] + U * d.abs()
    e_var = (depth(D) + 4) * U * var + (2 * d.abs() * e_d + e_d * e_d).mean(1)
    e_rstd = e_var / (var + eps) + 4 * U          # (half of it to first order)
    e_y = w.double().abs() * rstd[:, None] * (e_d + d.abs() * (e_rstd[:, None] + 4 * U)) + 2 * U * (y.abs() + bias.abs())
    return h, mean, rstd, y, e_mean, e_rstd, e_y


def check_norm(n, case, eps, quantize, what):
    xs, w, b, r = case
    h, mean, rstd, y, e_mean, e_rstd, e_y = norm_reference(xs, w, b, r, eps)
    tail = BF16 if xs.dtype == torch.bfloat16 else U
    within(host(n.mean), mean, e_mean + U * mean.abs(), what + " mean")
    within(host(n.rstd), rstd, e_rstd * rstd, what + " rstd")
    if r is not None:
        assert n.residual.dtype == xs.dtype
        within(host(n.residual), h, tail * h.abs() + U * (xs.double().abs() + r.double().abs()), what + " sum")
    if quantize:
        assert n.out.dtype == torch.float8_e4m3fn and n.scale.shape == (xs.shape[0], -(-xs.shape[1] // 128))
        # (the largest of a block is off by its own error at most)
        rel = (e_y / y.abs().clamp_min(1e-30)).clamp_max(1)
        block = y.abs() > 0.01 * y.abs().max()
        worst = rel[block].max().item() if bool(block.any()) else 0.0
        scale = host(n.scale).repeat_interleave(128, 1)[:, :y.shape[1]]
        got = host(n.out.float()) * scale
        within(got, y, y.abs() * (2.0 ** -4 + 8 * U) + 2 * e_y + scale * 2.0 ** -10, what)
        for i in range(0, y.shape[1], 128):
            top = y[:, i:i + 128].abs().amax(1)
            within(host(n.scale)[:, i // 128], (top / 448).clamp_min(2.0 ** -126),
                   (e_y[:, i:i + 128].amax(1) + 4 * U * top) / 448, what + " scale")
        assert worst < 1
    else:
        assert n.scale is None and n.out.dtype == xs.dtype
        within(host(n.out), y, tail * y.abs() + (1 + tail) * e_y, what)


@pytest.mark.parametrize("quantize", [False, True])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T,D", SIZES)
def test_layernorm(T, D, dtype, quantize):
    for residual in (False, True):
        case = norm_case(T, D, dtype, residual, 10 * D + T)
        xs, w, b, r = case
        for odd in (False, True):
            what = "layernorm %s" % ((T, D, dtype, quantize, residual, odd),)
            say(what)
            n = x.layernorm(dev(xs, odd), dev(w), dev(b), None if r is None else dev(r, odd), eps=1e-5, quantize=quantize)
            check_norm(n, case, 1e-5, quantize, what)


def test_layernorm_without_bias_and_weight_in_32_bits():
    xs, _, _, _ = norm_case(6, 300, "bf16", False, 1)
    xs[2] = 0
    xs[3] = 1.5                                   # a row without variance
    w, b = (1 + 0.2 * normal(2, 300)).float(), normal(3, 300).float()
    for bias in (None, b):
        n = x.layernorm(dev(xs), dev(w), None if bias is None else dev(bias), eps=1e-5)
        assert n.residual.data_ptr() is not None and torch.equal(n.residual.cpu(), xs)
        check_norm(n, (xs, w, bias, None), 1e-5, False, "fp32 weight")
        rows = host(n.out)[2:4]
        want = torch.zeros(300) if bias is None else bias
        assert torch.equal(rows, want.bfloat16().double().expand(2, 300))


@pytest.mark.parametrize("D", [1024, 20001])
def test_layernorm_of_rows_far_from_zero(D):
    """A mean a thousand times the spread: a variance from the sum of squares would be wrong in its first digit."""
    xs = (1000 + normal(4, 5, D)).float()
    w, b = torch.ones(D), torch.zeros(D)
    n = x.layernorm(dev(xs), dev(w), dev(b), eps=0.0)
    check_norm(n, (xs, w, b, None), 0.0, False, "far")
    _, _, rstd, _, _, _, _ = norm_reference(xs, w, b, None, 0.0)
    within(host(n.rstd), rstd, 0.02 * rstd, "rstd")


def test_layernorm_not_finite_values_stay_in_their_row():
    xs = normal(3, 5, 260).float()
    xs[1, 7], xs[3, 130] = float("nan"), float("inf")
    w, b = torch.ones(260), torch.zeros(260)
    for quantize in (False, True):
        n = x.layernorm(dev(xs), dev(w), dev(b), quantize=quantize)
        bad = torch.isnan(n.out.float()).cpu()
        assert bool(bad[1].all()) and bool(bad[3].all()) and not bool(bad[[0, 2, 4]].any())
        assert bool(torch.isnan(n.rstd.cpu()[[1, 3]]).all())


def test_layernorm_of_rows_without_columns():
    n = x.layernorm(torch.empty(3, 0, device="cuda"), torch.empty(0, device="cuda"), torch.empty(0, device="cuda"))
    assert n.out.shape == (3, 0) and bool(torch.isnan(n.mean).all()) and bool(torch.isnan(n.rstd).all())
    n = x.layernorm(torch.empty(0, 8, device="cuda"), torch.ones(8, device="cuda"))
    assert n.out.shape == (0, 8) and n.mean.shape == n.rstd.shape == (0,)


def backward_reference(dy, xs, w, mean, rstd, dr):
    T, D = xs.shape
    dy, xs, w, mean, rstd = dy.double(), xs.double(), w.double(), mean.double()[:, None], rstd.double()[:, None]
    xh, g = (xs - mean) * rstd, dy * w
    one, two = g.mean(1, keepdim=True), (g * xh).mean(1, keepdim=True)
    dx = rstd * (g - one - xh * two) + (dr.double() if dr is not None else 0)
    e_xh = 2 * U * (xs.abs() + mean.abs()) * rstd + 2 * U * xh.abs()
    n = depth(D) + 8
    e_dx = rstd * (8 * U * g.abs() + n * U * g.abs().mean(1, keepdim=True) + e_xh * two.abs()
                   + xh.abs() * (n * U * (g * xh).abs().mean(1, keepdim=True) + (g.abs() * e_xh).mean(1, keepdim=True)))
    e_dx = e_dx + 8 * U * (dx.abs() + (dr.double().abs() if dr is not None else 0))
    e_dw = (T + 8) * U * (dy * xh).abs().sum(0) + (dy.abs() * e_xh).sum(0)
    return dx, (dy * xh).sum(0), dy.sum(0), e_dx, e_dw, (T + 8) * U * dy.abs().sum(0)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T,D", [(0, 64), (1, 1), (1, 4096), (3, 129), (600, 40), (1030, 257), (37, 2050), (513, 1024),
                                 (270, 5001), (9, 8192), (2, 20001), (9001, 40), (2501, 1100), (2301, 2100), (601, 5001),
                                 (1201, 8200), (256, 2300), (2100, 4500), (300, 16500)])
def test_layernorm_backward(T, D, dtype):
    for residual in (False, True):
        xs, w, _, _ = norm_case(T, D, dtype, False, 7 * D + T)
        dy = as_type(normal(D, T, D), dtype)
        dr = as_type(normal(D + 1, T, D), dtype) if residual else None
        mean = xs.double().mean(1)
        rstd = (1 / torch.sqrt((xs.double() - mean[:, None]).square().mean(1) + 1e-5)).float()
        mean = mean.float()
        dx, dw, db, e_dx, e_dw, e_db = backward_reference(dy, xs, w, mean, rstd, dr)
        tail = BF16 if dtype == "bf16" else U
        for odd in (False, True):
            what = "layernorm_backward %s" % ((T, D, dtype, residual, odd),)
            say(what)
            gx, gw, gb = x.layernorm_backward(dev(dy, odd), dev(xs, odd), dev(w), dev(mean), dev(rstd),
                                              None if dr is None else dev(dr, odd))
            assert gx.dtype == xs.dtype and gw.dtype == gb.dtype == torch.float32
            within(host(gx), dx, tail * dx.abs() + (1 + tail) * e_dx, what + " dx")
            within(host(gw), dw, e_dw, what + " dweight")
            within(host(gb), db, e_db, what + " dbias")


@pytest.mark.parametrize("D,value", [(1, 2.0 ** 120), (100, 2.0 ** 113), (1001, 2.0 ** 113), (5001, 2.0 ** 113),
                                     (8201, 2.0 ** 113)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_layernorm_of_equal_large_values(D, value, dtype):
    """Powers of two whose sum of D is in fp32 and exact, but not their product with rstd = 1e6: centred they are 0."""
    xs = as_type(torch.full((3, D), value, dtype=torch.float64), dtype)
    xs[1] = 0
    w, b = as_type(1 + 0.2 * normal(2, D), dtype), as_type(0.5 * normal(5, D), dtype)
    dy = as_type(normal(6, 3, D), dtype)
    n = x.layernorm(dev(xs), dev(w), dev(b), eps=1e-12)
    assert torch.equal(host(n.out), b.double().expand(3, D))
    assert torch.equal(host(n.mean), torch.tensor([value, 0, value], dtype=torch.float64))
    rstd = n.rstd.cpu()
    within(rstd.double(), torch.full((3,), 1e6, dtype=torch.float64), 4 * U * 1e6, "rstd")
    gx, gw, gb = x.layernorm_backward(dev(dy), dev(xs), dev(w), n.mean, n.rstd)
    g = dy.double() * w.double()
    dx = rstd.double()[:, None] * (g - g.mean(1, keepdim=True))
    e = rstd.double()[:, None] * (4 * U * g.abs() + (depth(D) + 8) * U * g.abs().mean(1, keepdim=True)) + 4 * U * dx.abs()
    tail = BF16 if dtype == "bf16" else U
    within(host(gx), dx, tail * dx.abs() + (1 + tail) * e, "dx")
    assert not bool(gw.any())
    within(host(gb), dy.double().sum(0), 4 * U * dy.double().abs().sum(0), "dbias")


def test_layernorm_backward_against_differences():
    """Central differences of the 64-bit forward along random directions: their own error is about step^2."""
    T, D, eps, step = 9, 333, 1e-5, 1e-5
    xs, w, b = (1 + normal(1, T, D)).float(), (1 + 0.3 * normal(2, D)).float(), normal(5, D).float()
    dy = normal(3, T, D).float()
    n = x.layernorm(dev(xs), dev(w), dev(b), eps=eps)
    grads = [host(t) for t in x.layernorm_backward(dev(dy), dev(xs), dev(w), n.mean, n.rstd)]

    def loss(*leaf):
        return (norm_reference(*leaf, None, eps)[3] * dy.double()).sum().item()

    leaf = [xs.double(), w.double(), b.double()]
    for seed in range(4):
        for i, g in enumerate(grads):
            v = normal(20 + 10 * i + seed, *leaf[i].shape)
            up, down = list(leaf), list(leaf)
            up[i], down[i] = leaf[i] + step * v, leaf[i] - step * v
            num = (loss(*up) - loss(*down)) / (2 * step)
            assert abs(num - (g * v).sum().item()) <= 1e-4 * (g * v).norm().item() * 10


def test_layernorm_backward_gives_the_same_bits_again():
    xs, w, b, _ = norm_case(777, 1030, "bf16", False, 5)
    dy = dev(as_type(normal(6, 777, 1030), "bf16"))
    n = x.layernorm(dev(xs), dev(w), dev(b))
    first = x.layernorm_backward(dy, dev(xs), dev(w), n.mean, n.rstd)
    for _ in range(3):
        again = x.layernorm_backward(dy, dev(xs), dev(w), n.mean, n.rstd)
        assert all(torch.equal(p, q) for p, q in zip(first, again))


# ------------------------------------------------------------ linear layer

ACTS = [None, "relu", "gelu", "gelu_tanh", "silu"]
C2 = 2 * math.sqrt(2 / math.pi)


def act_reference(z, act):
    """The activation and its derivative in 64 bits, and how far the kernel's fp32 values of both may be off for an exact z.

    2^(x log2 e): the product and the constant round (2u |x|), the instruction by 2u; 1 / (1 + e) is a reciprocal
    (2u) of a rounded sum; six roundings make gelu_tanh's argument.  erff is within 16 steps."""
    if act is None:
        return z, torch.ones_like(z), torch.zeros_like(z), torch.zeros_like(z)
    if act == "relu":
        return z.clamp_min(0), (z > 0).double(), torch.zeros_like(z), torch.zeros_like(z)
    if act == "gelu":
        cdf, pdf = torch.special.ndtr(z), torch.exp(-0.5 * z * z) / math.sqrt(2 * math.pi)
        return (z * cdf, cdf + z * pdf, 20 * U * z.abs(),
                20 * U + z.abs() * pdf * (8 * U + 4 * U * z * z))
    arg = z if act == "silu" else C2 * z * (1 + 0.044715 * z * z)
    darg = torch.ones_like(z) if act == "silu" else C2 * (1 + 3 * 0.044715 * z * z)
    q = torch.sigmoid(arg)
    e_q = q * ((1 - q) * (8 * U * arg.abs() + 4 * U) + 4 * U) + 2.0 ** -126
    return (z * q, q + z * q * (1 - q) * darg, z.abs() * e_q + 2 * U * (z * q).abs(),
            e_q * (1 + z.abs() * darg) + 10 * U * (q + z.abs() * q * darg))


def linear_reference(a, b, bias, r, act, splits=16):
    """z and the layer's result in 64 bits, and how far the kernel's unrounded ones may be off."""
    a, b = a.double(), b.double()
    K = a.shape[1]
    z = a @ b
    e_z = 2 * U * (K + 8 + splits) * (a.abs() @ b.abs())
    if bias is not None:
        z = z + bias.double()
        e_z = e_z + 2 * U * (z.abs() + bias.double().abs())
    y, _, e_act, _ = act_reference(z, act)
    e_y = 1.13 * e_z + e_act + U * y.abs()               # no activation is steeper than 1.13
    if r is not None:
        y = y + r.double()
        e_y = e_y + U * (y.abs() + r.double().abs())
    return z, y, e_z, e_y


def linear_case(T, N, K, seed, scale=1.0):
    a = as_type(normal(seed, T, K), "bf16")
    b = as_type(scale * normal(seed + 1, K, N) / math.sqrt(max(K, 1)), "bf16")
    return a, b, normal(seed + 2, N), 2 * normal(seed + 3, T, N)


LAYERS = [(1, 1, 1), (1, 64, 64), (3, 5, 7), (1, 4096, 512), (7, 130, 129), (16, 256, 512), (17, 129, 1000), (33, 72, 136),
          (64, 64, 64), (5, 1000, 2047), (100, 300, 640), (65, 512, 2048), (130, 264, 1032), (257, 513, 384), (300, 1024, 256)]


@pytest.mark.parametrize("transpose_b", [False, True])
@pytest.mark.parametrize("T,N,K", LAYERS)
def test_linear(T, N, K, transpose_b):
    a, b, bias, r = linear_case(T, N, K, T + N + K)
    stored = b.t().contiguous() if transpose_b else b
    for i, act in enumerate(ACTS):
        out, other = ("f32", "bf16") if i % 2 else ("bf16", "f32")
        bias_t, r_t = as_type(bias, other), as_type(r, out if i < 3 else other)
        for odd in (False, True):
            what = "linear %s" % ((T, N, K, transpose_b, act, out, odd),)
            say(what)
            z, y, e_z, e_y = linear_reference(a, b, bias_t, r_t, act)
            got, kept = x.linear(dev(a, odd), dev(stored, odd), bias=dev(bias_t), residual=dev(r_t, odd), activation=act,
                                 transpose_b=transpose_b, keep=True, dtype=torch.float32 if out == "f32" else torch.bfloat16)
            tail = BF16 if out == "bf16" else U
            assert got.dtype == kept.dtype == (torch.float32 if out == "f32" else torch.bfloat16)
            within(host(got), y, tail * y.abs() + (1 + tail) * e_y, what)
            within(host(kept), z, tail * z.abs() + (1 + tail) * e_z, what + " z")
    z, y, e_z, e_y = linear_reference(a, b, None, None, None)
    got = x.linear(dev(a), dev(stored), transpose_b=transpose_b)
    assert got.dtype == torch.float32
    within(host(got), y, e_y + U * y.abs(), "nothing but the product")


@pytest.mark.parametrize("T,N,K", [(0, 5, 8), (4, 0, 8), (3, 5, 0), (0, 0, 0)])
def test_linear_empty(T, N, K):
    a, b, bias, r = linear_case(T, N, K, 3)
    for turned in (False, True):
        got, z = x.linear(dev(a), dev(b.t().contiguous() if turned else b), dev(bias.float()), dev(r.float()), "silu", turned, True)
        assert got.shape == z.shape == (T, N)
        if K == 0 and T and N:
            want = bias.float().double()
            within(host(z), want.expand(T, N), U * want.abs(), "bias alone")
    dw = x.linear_wgrad(dev(a), dev(as_type(r, "bf16")))
    assert dw.shape == (K, N) and (T or not bool(dw.any()))
    dz, db = x.activation_backward(dev(r.float()), dev(r.float()), "gelu")
    assert dz.shape == (T, N) and db.shape == (N,) and (T or not bool(db.any()))


def test_linear_writes_its_own_columns_only():
    for T, N, K in ((37, 150, 200), (3, 30, 2048), (300, 261, 400)):
        a, b, bias, _ = linear_case(T, N, K, 11)
        bias = bias.float()
        for dtype in (torch.float32, torch.bfloat16):
            wide = torch.full((T, N + 13), 5.0, device="cuda", dtype=dtype)
            got = x.linear(dev(a), dev(b), dev(bias), activation="relu", out=wide[:, 3:N + 3])
            _, y, _, e = linear_reference(a, b, bias, None, "relu")
            tail = BF16 if dtype == torch.bfloat16 else U
            within(host(got), y, tail * y.abs() + (1 + tail) * e, "out")
            assert bool((wide[:, :3] == 5).all()) and bool((wide[:, N + 3:] == 5).all())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T,N,K", [(1, 4096, 4096), (5, 77, 130), (300, 520, 264), (1531, 2000, 4096)])
def test_linear_adds_to_its_residual_in_place(T, N, K, dtype):
    a, b, bias, r = linear_case(T, N, K, 5, 1 / 16)
    a, b, bias, r = dev(a), dev(b), dev(as_type(bias, "f32")), dev(as_type(r, dtype))
    apart = x.linear(a, b, bias, r, "silu", dtype=r.dtype)
    assert x.linear(a, b, bias, r, "silu", out=r) is r
    assert torch.equal(apart, r)


@pytest.mark.parametrize("T", [3, 200])
def test_linear_nan_stays_in_its_row_and_column(T):
    """A NaN behind the end of k, or in another row, does not reach a result; relu keeps it."""
    K, N = 136, 140
    a, b, bias, _ = linear_case(T, N, K + 16, 5)
    a[:, K:], b[K:] = float("nan"), float("nan")
    a[1, 5], b[130, 77] = float("nan"), float("nan")
    for turned in (False, True):
        stored = b.t().contiguous() if turned else b
        stored = dev(stored)[:, :K] if turned else dev(stored)[:K]
        got = host(x.linear(dev(a)[:, :K], stored, dev(bias.float()), activation="relu", transpose_b=turned))
        bad = torch.isnan(got)
        assert bool(bad[1].all()) and bool(bad[:, 77].all()) and int(bad.sum()) == T + N - 1


@pytest.mark.parametrize("T,N,K", [(1, 1, 1), (3, 5, 7), (64, 64, 64), (1000, 130, 72), (129, 264, 136), (2048, 64, 128),
                                   (4099, 40, 264), (2047, 129, 70), (600, 1032, 520)])
def test_linear_wgrad(T, N, K):
    a, dy = as_type(normal(K, T, K), "bf16"), as_type(normal(N, T, N), "bf16")
    ref, mag = a.double().t() @ dy.double(), a.double().abs().t() @ dy.double().abs()
    for out in (torch.float32, torch.bfloat16):
        for odd in (False, True):
            say("linear_wgrad", T, N, K, out, odd)
            got = x.linear_wgrad(dev(a, odd), dev(dy, odd), dtype=out)
            tail = BF16 if out == torch.bfloat16 else U
            within(host(got), ref, 2 * U * (T + 24) * mag + tail * ref.abs(), "linear_wgrad")


@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("T,N", [(1, 1), (3, 7), (5, 512), (600, 130), (33, 1021), (128, 1100), (129, 1100), (2049, 520), (9000, 40)])
def test_activation_backward(T, N, act):
    for dy_t, z_t in (("bf16", "bf16"), ("f32", "f32"), ("f32", "bf16")):
        dy, z = as_type(normal(T, T, N), dy_t), as_type(3 * normal(N, T, N), z_t)
        _, slope, _, e = act_reference(z.double(), act)
        ref, off = dy.double() * slope, dy.double().abs() * e + U * (dy.double() * slope).abs()
        for odd in (False, True):
            say("activation_backward", T, N, act, dy_t, z_t, odd)
            dz, db = x.activation_backward(dev(dy, odd), dev(z, odd), act)
            assert dz.dtype == torch.bfloat16 and db.dtype == torch.float32
            within(host(dz), ref, BF16 * ref.abs() + (1 + BF16) * off + 2.0 ** -133, "dz")
            within(host(db), ref.sum(0), (T + 8) * U * ref.abs().sum(0) + off.sum(0), "dbias")


@pytest.mark.parametrize("act", ACTS[1:])
def test_activations_far_from_zero(act):
    """Large, infinite and NaN arguments: the limits, and no NaN where there is a limit."""
    v = torch.tensor([[-3e38, -1e4, -90.0, -20.0, -0.0, 0.0, 20.0, 90.0, 1e4, 3e37, float("inf"), float("nan")]])
    one = torch.ones(1, 1).bfloat16()
    got = host(x.linear(dev(one), dev(torch.zeros(1, 12).bfloat16()), dev(v[0]), activation=act))[0]
    _, slopes = None, host(x.activation_backward(dev(torch.ones(1, 12)), dev(v), act)[0])[0]
    assert bool((got[:3].abs() < 1e-30).all()) and bool((slopes[:3].abs() < 1e-30).all())
    assert torch.equal(got[7:11], v[0, 7:11].double()) and bool((slopes[7:10] == 1).all())
    assert bool(torch.isnan(got[11])) and bool(torch.isnan(slopes[11]))
    assert abs(got[4].item()) == abs(got[5].item()) == 0


@pytest.mark.parametrize("act", ACTS)
def test_linear_gradients_against_differences(act):
    """Central differences of the 64-bit layer: the operands of the products are bf16, so is dz."""
    T, N, K, step = 19, 40, 72, 1e-5
    a, b, bias, r = linear_case(T, N, K, 8)
    bias, dout = bias.float(), as_type(normal(9, T, N), "bf16")
    _, z = x.linear(dev(a), dev(b), dev(bias), dev(r.float()), act, keep=True)
    dz, db = x.activation_backward(dev(dout), z, act)
    da, dw, dwt = (host(g) for g in (x.linear(dz, dev(b), transpose_b=True), x.linear_wgrad(dev(a), dz),
                                     x.linear_wgrad(dz, dev(a))))
    d, p, q = host(dz).abs(), a.double().abs(), b.double().abs()
    within(dwt.t(), dw, 4 * U * (T + 24) * (p.t() @ d), "the weights' gradient of the other layout")

    def loss(*leaf):
        return (act_reference(leaf[0] @ leaf[1] + leaf[2], act)[0] * dout.double()).sum().item()

    # dz is rounded once (2^-8 of each value); the differences' own error is far below that
    leaf = [a.double(), b.double(), bias.double()]
    for i, (g, mag) in enumerate(((da, d @ q.t()), (dw, p.t() @ d), (host(db), d.sum(0)))):
        for seed in range(3):
            v = normal(40 + 10 * i + seed, *leaf[i].shape)
            up, down = list(leaf), list(leaf)
            up[i], down[i] = leaf[i] + step * v, leaf[i] - step * v
            num = (loss(*up) - loss(*down)) / (2 * step)
            assert abs(num - (g * v).sum().item()) <= 1.5 * BF16 * (mag * v.abs()).sum().item()


# ---------------------------- streams, graphs, far offsets, the two ways of a call


def chain(v, w, r):
    """The operators as a block uses them, from rows ``v`` [T, 256]: everything that they give."""
    n = x.layernorm(v, w["norm"], w["bias"], v)
    route = x.route_experts(x.linear(n.out, w["router"], transpose_b=True), 3, r)
    y, z = x.linear(n.out, w["v1"], w["c1"], activation="gelu", keep=True, dtype=torch.bfloat16)
    rows = n.out[route.token.clamp_min(0)]
    out = x.combine_experts(rows, route.row, route.p, residual=x.linear(y, w["v2"], w["c2"], residual=n.residual))
    drows, dp = x.combine_experts_backward(v, rows, route.row, route.token, route.p)
    ds = x.route_experts_backward(dp, x.linear(n.out, w["router"], transpose_b=True), route.expert, route.p, route.counts, 0.1)
    dz, dc = x.activation_backward(x.linear(v, w["v2"], transpose_b=True, dtype=torch.bfloat16), z, "gelu")
    dn = x.linear(dz, w["v1"], transpose_b=True, residual=x.combine_experts(drows, route.row), dtype=torch.bfloat16)
    return [*n[:1], *n[2:], *route, y, z, out, drows, dp, ds, dz, dc, x.linear_wgrad(n.out, dz), dn,
            *x.layernorm_backward(dn, n.residual, w["norm"], n.mean, n.rstd)]


def chain_weights(D=256, S=320, E=12):
    w = {"norm": 1 + 0.1 * normal(1, D), "bias": 0.1 * normal(2, D), "router": normal(3, E, D) / 16, "v1": normal(4, D, S) / 16,
         "c1": normal(5, S), "v2": normal(6, S, D) / 18, "c2": normal(7, D)}
    return {k: t.bfloat16().cuda() for k, t in w.items()}


@pytest.mark.parametrize("T", [1, 33, 700])
def test_captured_in_a_graph(T):
    """Replays give what eager calls give, with new values in the same tensors and eager work between them."""
    w, v, there = chain_weights(), normal(8, T, 256).bfloat16().cuda(), torch.ones(T, dtype=torch.bool, device="cuda")
    chain(v, w, there)
    torch.cuda.synchronize()
    graph, other = torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = chain(v, w, there)
    u = v.clone()
    with torch.cuda.graph(other):
        second = chain(u, w, there)
    for seed in range(4):
        v.copy_(normal(10 + seed, T, 256).bfloat16())
        u.copy_(normal(20 + seed, T, 256).bfloat16())
        there.copy_(torch.rand(T, generator=torch.Generator().manual_seed(seed)) < (0.8 if seed < 3 else 0))
        graph.replay()
        other.replay()
        want = chain(v, w, there), chain(u, w, there)
        torch.cuda.synchronize()
        for a, b in zip(captured + second, want[0] + want[1]):
            assert torch.equal(torch.nan_to_num(a), torch.nan_to_num(b))


def test_operators_run_on_the_current_stream():
    """Each call is enqueued behind what the current stream holds, and before what follows on it."""
    w, src = chain_weights(), normal(1, 300, 256).bfloat16().cuda()
    want = [t.clone() for t in chain(src, w, None)]
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        torch.cuda._sleep(20_000_000)
        got = chain(src * 1, w, None)
        after = [t * 1 for t in got]
    s.synchronize()
    for p, q in zip(want, after):
        assert torch.equal(p, q)


def test_native_and_python_paths_agree(monkeypatch):
    """The plain calls go through the native module; without it the same library is called from Python."""
    w, v, there = chain_weights(), normal(1, 300, 256).bfloat16().cuda(), (normal(2, 300) < 0.5).cuda()
    assert x._fast is not None
    taken = []
    for name in ("layernorm", "layernorm_backward", "linear", "linear_wgrad", "activation_backward", "route_experts",
                 "route_experts_backward", "combine_experts", "combine_experts_backward"):
        def counted(*args, f=getattr(x._fast, name), name=name):
            r = f(*args)
            taken.append((name, r is not None))
            return r
        monkeypatch.setattr(x._fast, name, counted)
    q = x.layernorm(v, w["norm"], quantize=True)
    native = [t.clone() for t in chain(v, w, there)] + [q.out.float(), q.scale]
    out = torch.empty(300, 320, dtype=torch.bfloat16, device="cuda")
    assert x.linear(v, w["v1"], out=out) is out and x.linear(v, w["v1"], out=out, keep=True)[0] is out
    native += [out.clone(), x.linear_wgrad(v, v, dtype=torch.bfloat16), x.activation_backward(v, v, None)[1]]
    assert len({n for n, _ in taken}) == 9 and all(ok for _, ok in taken)
    monkeypatch.setattr(x, "_fast", None)
    q = x.layernorm(v, w["norm"], quantize=True)
    python = chain(v, w, there) + [q.out.float(), q.scale]
    assert x.linear(v, w["v1"], out=out) is out
    python += [out.clone(), x.linear_wgrad(v, v, dtype=torch.bfloat16), x.activation_backward(v, v, None)[1]]
    for a, b in zip(native, python):
        assert a.dtype == b.dtype and a.shape == b.shape and torch.equal(a, b)


def test_rows_past_32_bit_offsets():
    """Operands of more than 2^32 bytes: the last rows are the right ones."""
    T, D = 600_000, 4096
    a = torch.zeros(T, D, dtype=torch.bfloat16, device="cuda")               # 4.9 GB
    last = as_type(normal(2, 40, D), "bf16")
    a[-40:] = last.cuda()
    w = as_type(1 + 0.1 * normal(3, D), "bf16")
    n = x.layernorm(a, w.cuda(), None, a)
    _, mean, rstd, y, e_mean, e_rstd, e_y = norm_reference(last, w, None, last, 1e-5)
    within(host(n.out[-40:]), y, BF16 * y.abs() + (1 + BF16) * e_y, "layernorm")
    del n
    b, bias = as_type(normal(4, D, 64) / 64, "bf16"), as_type(normal(5, 64), "bf16")
    z, ref, e_z, e = linear_reference(last, b, bias, None, "silu")
    got = x.linear(a, b.cuda(), bias.cuda(), activation="silu")
    within(host(got[-40:]), ref, e + U * ref.abs(), "linear")
    dw = x.linear_wgrad(a, torch.cat([torch.zeros(T - 40, 64, dtype=torch.bfloat16), as_type(normal(6, 40, 64), "bf16")]).cuda())
    p, q = last.double(), as_type(normal(6, 40, 64), "bf16").double()
    within(host(dw), p.t() @ q, 2 * U * 64 * (p.abs().t() @ q.abs()) + U * (p.t() @ q).abs(), "linear_wgrad")
    dz, db = x.activation_backward(a, a, "relu")
    ref = last.double().clamp_min(0)
    within(host(dz[-40:]), ref, BF16 * ref, "dz")
    within(host(db), ref.sum(0), 48 * U * ref.sum(0), "dbias")
    del dz
    row = torch.full((3, 2), T - 40, dtype=torch.int32) + torch.arange(6).view(3, 2).int()
    got = x.combine_experts(a, row.cuda())
    ref = last.double()[:6].view(3, 2, D).sum(1)
    within(host(got), ref, 4 * U * last.double()[:6].abs().view(3, 2, D).sum(1), "combine")


def test_refusals_on_the_gpu():
    def c(*shape, dtype=torch.bfloat16):
        return torch.zeros(*shape).to(dtype).cuda()

    f32, i32 = torch.float32, torch.int32
    cases = [
        (lambda: x.layernorm(c(4, 8), c(9)), ValueError, "weight must be a contiguous vector of 8"),
        (lambda: x.layernorm(c(4, 8), c(8), c(8, dtype=f32)), TypeError, "bias must be bfloat16"),
        (lambda: x.layernorm(c(4, 8), c(8), None, c(4, 9)), ValueError, "residual must be"),
        (lambda: x.layernorm(c(4, 8), c(8), eps=-1.0), x.XtcError, "extent|shape"),
        (lambda: x.layernorm_backward(c(4, 8), c(4, 8), c(8), c(4), c(4, dtype=f32)), TypeError, "mean must be float32"),
        (lambda: x.linear(c(4, 8), c(9, 4)), ValueError, "inner dimensions differ"),
        (lambda: x.linear(c(4, 8), c(4, 9), transpose_b=True), ValueError, "inner dimensions differ"),
        (lambda: x.linear(c(4, 8), c(8, 4), c(5)), ValueError, "bias must be a contiguous vector of 4"),
        (lambda: x.linear(c(4, 8), c(8, 4), None, c(4, 5)), ValueError, "residual must be"),
        (lambda: x.linear(c(4, 8), c(8, 4), dtype=torch.float16), TypeError, "dtype must be"),
        (lambda: x.linear(c(4, 8), c(8, 4), out=c(4, 5)), ValueError, "out must be"),
        (lambda: x.linear(c(1, 8).expand(4, 8), c(8, 4)), x.XtcError, "leading|stride"),
        (lambda: x.linear(c(4, 8), c(4, 8).t()), ValueError, "unit stride"),
        (lambda: x.linear_wgrad(c(4, 8), c(5, 4)), ValueError, "rows"),
        (lambda: x.activation_backward(c(4, 8), c(4, 9), "silu"), ValueError, "z must be"),
        (lambda: x.route_experts(c(4, 8), 9), ValueError, "top must be"),
        (lambda: x.route_experts(c(4, 8), 0), ValueError, "top must be"),
        (lambda: x.route_experts(c(4, 64), 17), x.XtcError, "too large"),
        (lambda: x.route_experts(c(4, 2000), 2), x.XtcError, "too large"),
        (lambda: x.route_experts(c(4, 8), 2, c(4)), TypeError, "mask must be bool"),
        (lambda: x.route_experts(c(4, 8), 2, c(5).bool()), ValueError, "mask must be"),
        (lambda: x.route_experts_backward(None, c(4, 8), c(4, 2, dtype=i32), c(4, 2, dtype=f32), c(9, dtype=i32)),
         ValueError, "counts must be"),
        (lambda: x.route_experts_backward(c(4, 2), c(4, 8), c(4, 2, dtype=i32), c(4, 2, dtype=f32), c(8, dtype=i32)),
         TypeError, "dp must be float32"),
        (lambda: x.combine_experts(c(8, 8), c(4, 2)), TypeError, "row must be int32"),
        (lambda: x.combine_experts(c(8, 8), c(4, 2, dtype=i32), c(4, 3, dtype=f32)), ValueError, "p must be"),
        (lambda: x.combine_experts(c(8, 8), c(4, 2, dtype=i32), None, c(4, 9)), ValueError, "residual must be"),
        (lambda: x.combine_experts_backward(c(4, 8), c(9, 8), c(4, 2, dtype=i32), c(8, dtype=i32), c(4, 2, dtype=f32)),
         ValueError, "rows must hold 8 rows"),
        (lambda: x.combine_experts_backward(c(4, 9), c(8, 8), c(4, 2, dtype=i32), c(8, dtype=i32), c(4, 2, dtype=f32)),
         ValueError, "dout must be"),
    ]
    for make, error, match in cases:
        with pytest.raises(error, match=match):
            make()

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
                                 (1201, 8200)])
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

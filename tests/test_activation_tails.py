"""The activations and their derivatives far from zero, relative to their own values, against their definitions in
64 bits.

Tolerances, u = 2^-24.  gelu is v times a normal distribution that left of zero is e^(-v^2 / 2) times a polynomial in
t = 1 / (1 + 0.35 |v|), right of zero 1 less as much.  v^2 / 2 rounds, e^x as 2^(x log2 e) twice more (3u x in all), the
instruction by 2u; t by 3u, which its function follows at most one for one; the polynomial is fitted within u, and its
eight steps round what is at most 2.2 times their sum (5u); two products and a difference: (1.5 v^2 + 16) u.  Its
derivative's other term is v times the same density, by three products.  silu and gelu_tanh pass one exponential,
whose argument x rounds seven times at most and twice more on the way to base 2 (9u |x| (1 - q) of a logistic q), a sum
(u) and a reciprocal (2u); the derivative's second term has eleven roundings more.  An exponential or a logistic below
2^-126 may be zero, before its products."""
import math

import pytest

from _helpers import say
from test_operators import BF16, U, dev, host, within

torch = pytest.importorskip("torch")
x = pytest.importorskip("paper_2512_16512_amd")

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU visible")


C2 = 2 * math.sqrt(2 / math.pi)
SWEEPS = {"left": torch.linspace(-12, -3, 4099), "middle": torch.linspace(-3, 3, 2051), "right": torch.linspace(3, 12, 513),
          "beyond": torch.linspace(-40, -12, 1025)}


def reference(v, act):
    """The activation and its derivative in 64 bits, and how far off fp32 values of them may be."""
    v, tiny = v.double(), 2.0 ** -126
    if act == "gelu":
        cdf, pdf = torch.special.erfc(-v / math.sqrt(2)) / 2, torch.exp(-0.5 * v * v) / math.sqrt(2 * math.pi)
        e_cdf = cdf * U * (1.5 * v * v + 16)
        y, slope = v * cdf, cdf + v * pdf
        return y, slope, v.abs() * (e_cdf + tiny) + 2 * U * y.abs(), \
            e_cdf + v.abs() * pdf * U * (1.5 * v * v + 6) + 2 * U * slope.abs() + tiny * (1 + v.abs())
    arg = v if act == "silu" else C2 * v * (1 + 0.044715 * v * v)
    darg = torch.ones_like(v) if act == "silu" else C2 * (1 + 3 * 0.044715 * v * v)
    q, other = torch.sigmoid(arg), torch.sigmoid(-arg)
    e_q = q * U * (9 * arg.abs() * other + 5) + tiny
    y, slope = v * q, q + v * q * other * darg
    e_slope = e_q + (v * darg).abs() * (e_q * (other + q) + 12 * U * q * other) + 2 * U * slope.abs()
    return y, slope, v.abs() * e_q + 2 * U * y.abs(), e_slope


@pytest.mark.parametrize("act", ["gelu", "gelu_tanh", "silu"])
@pytest.mark.parametrize("where", list(SWEEPS))
def test_activation(where, act):
    v = SWEEPS[where]
    n = v.shape[0]
    empty = torch.empty(3, 0, dtype=torch.bfloat16).cuda(), torch.empty(0, n, dtype=torch.bfloat16).cuda()
    y, _, e, _ = reference(v, act)
    for dtype, tail in ((torch.float32, U), (torch.bfloat16, BF16)):
        say("activation", act, where, dtype)
        got, z = x.linear(*empty, bias=dev(v), activation=act, keep=True, dtype=dtype)      # K = 0: act(bias)
        assert torch.equal(z.cpu(), v.to(dtype).expand(3, n))
        within(host(got), y.expand(3, n), (tail * y.abs() + (1 + tail) * e).expand(3, n), act)


@pytest.mark.parametrize("act", ["gelu", "gelu_tanh", "silu"])
@pytest.mark.parametrize("where", list(SWEEPS))
def test_derivative(where, act):
    v = SWEEPS[where]
    _, slope, _, e = reference(v, act)
    say("derivative", act, where)
    dz, db = x.activation_backward(torch.ones(1, v.shape[0]).cuda(), dev(v[None]), act)
    within(host(db), slope, e, act)           # (of one row: the products before their rounding)
    within(host(dz)[0], slope, BF16 * slope.abs() + (1 + BF16) * e, act)

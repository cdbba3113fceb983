"""Training steps of more experts, or more choices, than the routing operator takes: they train their router and have their
balance loss too, against the same block in 64 bits (tolerances as in test_moe_training)."""
import pytest

from _helpers import say
from test_moe import rel
from test_moe_training import block, make

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def moe():
    if not torch.cuda.is_available():
        pytest.skip("no GPU visible")
    from paper_2512_16512_amd import moe as mod
    return mod


@pytest.mark.parametrize("E,top", [(20, 17), (1100, 2), (1024, 16)])
def test_train_step_with_balance(moe, E, top):
    T, balance = 60, 3.0
    norm, router, w1, w2, x, r, dout, bias, _ = make(moe, T, 64, 48, 32, E)
    say("train step of", E, top)
    s = moe.train_step(x, r, norm, router, w1, w2, dout, top, bias=bias, balance=balance)
    n = moe._normed(x, norm, bias, r)
    route = moe.routing(moe.linear(n.out, router, transpose_b=True), top)
    assert (route.loss is None) == (E > 1024 or top > 16)
    h = moe.matmul_grouped(n.out[route.token], w1, route.ends, relu=True, dtype=torch.bfloat16)
    on = (h > 0).double().cpu()[route.row.cpu().long()]
    leaf = [t.double().cpu().requires_grad_() for t in (norm, router, w1, w2, bias)]
    h64 = (x.double().cpu() + r.double().cpu()).requires_grad_()
    out, loss = block(h64, leaf[0], leaf[4], *leaf[1:4], None, route.expert.cpu().long(), balance, top, on)
    ((out * dout.double().cpu()).sum() + loss).backward()
    assert rel(s.out, out.detach()) < 10 * 0.0017
    assert abs(s.loss.item() * balance - loss.item()) < 10 * 0.0017 * loss.item()
    for name, got, t in (("x", s.dx, h64), ("norm", s.dnorm, leaf[0]), ("router", s.drouter, leaf[1]),
                         ("w1", s.dw1, leaf[2]), ("w2", s.dw2, leaf[3]), ("bias", s.dbias, leaf[4])):
        assert rel(got, t.grad) < 10 * 0.0017, name


def test_torchs_loss_and_gradient_are_the_operators(moe):
    """On scores that both take, a row of -inf among them: the loss and the scores' gradient.  u = 2^-24; a softmax over E
    scores is within 8 u (1 + its spread), sums of T or E terms within T u or E u of their magnitudes."""
    T, E, top, u = 300, 40, 4, 2.0 ** -24
    g = torch.Generator().manual_seed(8)
    scores = torch.randn(T, E, generator=g).cuda()
    scores[7, 3:] = -torch.inf                              # (fewer than top left)
    dp = torch.randn(T, top, generator=g).cuda()
    r = moe.route_experts(scores, top)
    own = moe.route_experts_backward(dp, scores, r.expert, r.p, r.counts, 0.7)
    factor, q, c = moe._balance(scores, r.counts, top)
    assert bool(((factor * (c * q.sum(0)).sum() - r.loss).abs() <= 2 * (T + E + 100) * u * r.loss))
    wide = torch.cat([scores, torch.full((T, 1100 - E), -torch.inf, device="cuda")], 1)      # (never chosen, weight 0)
    more = r._replace(counts=torch.cat([r.counts, r.counts.new_zeros(1100 - E)]))
    got = moe.routing_backward(dp, wide, more, 0.7 * E / 1100, torch.float32)
    assert not bool(got[:, E:].any())
    size = 0.7 * factor * q * (c + (q * c).sum(1, keepdim=True))
    size = size.scatter_add(1, r.expert.long(), r.p * (dp.abs() + (r.p * dp).abs().sum(1, keepdim=True)))
    assert bool(((got[:, :E] - own).abs() <= 2 * (E + 200) * u * size).all())
    none = wide.clone()
    none[5] = -torch.inf
    assert not bool(moe._balance(none, more.counts, top)[1][5].any())

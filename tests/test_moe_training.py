"""The mixture-of-experts step that trains its router and an expert for every token, and the block on a layer norm:
the layer norm, linear, routing and combining operators run together, against the same block in 64 bits.

Tolerances, as relative Frobenius errors: a value rounded to bfloat16 is off by 0.17 %; ten roundings lie on the longest
way of the training step (those of the served one as in its other test: four of 2.6 %, allowed twice)."""
import pytest

from _helpers import say
from test_moe import rel

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def moe():
    if not torch.cuda.is_available():
        pytest.skip("no GPU visible")
    from paper_2512_16512_amd import moe as mod
    return mod


def make(moe, T, D=256, F=384, S=320, E=6, seed=11):
    norm, router, w1, w2 = moe.weights(E, D, F)
    g = torch.Generator().manual_seed(seed)

    def normal(*shape):
        return torch.randn(*shape, generator=g)

    x, r, dout = (normal(T, D).bfloat16().cuda() for _ in range(3))
    bias = (0.3 * normal(D)).bfloat16().cuda()
    shared = ((normal(D, S) / D ** 0.5).bfloat16().cuda(), (0.2 * normal(S)).cuda(), (normal(S, D) / S ** 0.5).bfloat16().cuda(),
              (0.2 * normal(D)).cuda())
    return norm, router, w1, w2, x, r, dout, bias, shared


def block(x, norm, bias, router, w1, w2, shared, expert, balance, top, on):
    """(out, balance loss) in 64 bits, differentiable, for the experts that the step chose; ``on``: which hidden values of
    its experts were above zero (see test_moe.block)."""
    T, E = x.shape[0], w1.shape[0]
    if bias is None:
        y = norm * x / torch.sqrt(x.square().mean(1, keepdim=True) + 1e-6)
    else:
        d = x - x.mean(1, keepdim=True)
        y = norm * d / torch.sqrt(d.square().mean(1, keepdim=True) + 1e-5) + bias
    scores = y @ router.t()
    p = torch.softmax(torch.gather(scores, 1, expert), 1)
    out = torch.zeros_like(y)
    for e in range(E):
        for j in range(top):
            at = (expert[:, j] == e).nonzero()[:, 0]
            out = out.index_add(0, at, p[at, j:j + 1] * ((y[at] @ w1[e]) * on[at, j]) @ w2[e])
    if shared is not None:
        v1, c1, v2, c2 = shared
        out = out + torch.nn.functional.gelu(y @ v1 + c1, approximate="tanh") @ v2 + c2
    counts = torch.bincount(expert.flatten(), minlength=E).double()
    return out, balance * E / (top * T * T) * (counts * torch.softmax(scores, 1).sum(0)).sum()


@pytest.mark.parametrize("with_bias,with_shared", [(False, True), (True, False), (True, True)])
def test_train_step_with_router(moe, with_bias, with_shared):
    T, top, balance = 300, 2, 3.0
    norm, router, w1, w2, x, r, dout, bias, shared = make(moe, T)
    bias, shared = bias if with_bias else None, shared if with_shared else None
    say("train step with router", with_bias, with_shared)
    s = moe.train_step(x, r, norm, router, w1, w2, dout, top, bias=bias, balance=balance, shared=shared)
    n = moe._normed(x, norm, bias, r)
    route = moe.routing(moe.linear(n.out, router, transpose_b=True), top)
    h = moe.matmul_grouped(n.out[route.token], w1, route.ends, relu=True, dtype=torch.bfloat16)
    on = (h > 0).double().cpu()[route.row.cpu().long()]
    leaf = [t.double().cpu().requires_grad_() for t in (norm, router, w1, w2)]
    h64 = (x.double().cpu() + r.double().cpu()).requires_grad_()
    b64 = bias.double().cpu().requires_grad_() if with_bias else None
    s64 = [t.double().cpu().requires_grad_() for t in shared] if with_shared else None
    out, loss = block(h64, leaf[0], b64, *leaf[1:], s64, route.expert.cpu().long(), balance, top, on)
    ((out * dout.double().cpu()).sum() + loss).backward()
    assert rel(s.out, out.detach()) < 10 * 0.0017
    assert abs(s.loss.item() * balance - loss.item()) < 10 * 0.0017 * loss.item()
    named = [("x", s.dx, h64), ("norm", s.dnorm, leaf[0]), ("router", s.drouter, leaf[1]), ("w1", s.dw1, leaf[2]),
             ("w2", s.dw2, leaf[3])]
    if with_bias:
        named.append(("bias", s.dbias, b64))
    if with_shared:
        named += zip(("v1", "c1", "v2", "c2"), s.dshared, s64)
    for name, got, t in named:
        assert rel(got, t.grad) < 10 * 0.0017, name
    assert (s.dbias is None) != with_bias and (s.dshared is None) != with_shared


@pytest.mark.parametrize("tokens", [1, 7, 200])
def test_served_step_on_a_layer_norm(moe, tokens):
    norm, router, w1, w2, x, r, _, bias, _ = make(moe, tokens)
    served = moe.Served(norm, router, w1, w2, bias=bias)
    say("served step on a layer norm", tokens)
    out, total = served.step(x, r)
    n = moe._normed(x, norm, bias, r, quantize=True)
    route = moe.routing(moe.matmul_fp8(n.out, n.scale, *served.router), 2)
    d = [t.double().cpu() for t in (x, r, norm, bias, w1, w2)]
    h = d[0] + d[1]
    c = h - h.mean(1, keepdim=True)
    y = d[2] * c / torch.sqrt(c.square().mean(1, keepdim=True) + 1e-5) + d[3]
    want = torch.zeros_like(y)
    for t in range(tokens):
        for j, e in enumerate(route.expert[t].tolist()):
            want[t] += route.p[t, j].item() * torch.relu(y[t] @ d[4][e]) @ d[5][e]
    assert rel(out, want) < 4 * 0.026 and rel(total, h) < 2 ** -8


def test_steps_with_router_give_the_same_bits_again_and_do_not_wait(moe):
    norm, router, w1, w2, x, r, dout, bias, shared = make(moe, 2000, 512, 128, 200, 16)
    args = dict(top=8, bias=bias, balance=0.5, shared=shared)
    first = moe.train_step(x, r, norm, router, w1, w2, dout, **args)
    torch.cuda.synchronize()
    torch.cuda.set_sync_debug_mode("error")
    try:
        again = moe.train_step(x, r, norm, router, w1, w2, dout, **args)
    finally:
        torch.cuda.set_sync_debug_mode("default")

    def flat(s):
        return [t for t in s if isinstance(t, torch.Tensor)] + list(s.dshared)

    for p, q in zip(flat(first), flat(again)):
        assert torch.equal(p, q)


def test_a_router_of_more_choices_than_the_operator_takes(moe):
    """Falls back to torch, with the same results."""
    T, E = 50, 40
    scores = torch.randn(T, E, generator=torch.Generator().manual_seed(1)).cuda()
    with pytest.raises(RuntimeError, match="too large"):
        moe.route_experts(scores, 20)
    r = moe.routing(scores, 20)
    v = torch.sort(scores, dim=1, descending=True, stable=True)
    assert torch.equal(r.expert.long(), v.indices[:, :20])
    assert torch.allclose(r.p, torch.softmax(v.values[:, :20], 1), rtol=1e-5)
    few = moe.routing(scores.double(), 4)       # (64 bits: torch's)
    own = moe.routing(scores, 4)
    for p, q in zip(few[:6], own[:6]):
        assert torch.allclose(p.double(), q.double(), rtol=1e-5), (p, q)
    token, ends, p, which = moe.route(scores.t().contiguous().t(), 4)
    assert torch.equal(token, own.token.long()) and torch.equal(ends, own.ends) and sorted(which.tolist()) == list(range(T * 4))


def test_steps_of_no_tokens_with_router(moe):
    norm, router, w1, w2, x, r, dout, bias, shared = make(moe, 0)
    s = moe.train_step(x, r, norm, router, w1, w2, dout, bias=bias, balance=1.0, shared=shared)
    assert s.out.shape == s.dx.shape == (0, 256) and s.loss.item() == 0
    for g, w in zip((s.drouter, s.dw1, s.dbias, *s.dshared), (router, w1, bias, *shared)):
        assert g.shape == w.shape and not bool(g.any())

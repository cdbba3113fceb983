"""What torch follows stays followed: the routing weights carry the gradient of scores that require one, a step's result that
of its router, and the routing can be traced and transformed.

Tolerances, u = 2^-24: a softmax over a token's choices is within 8 u (1 + s) of itself, s the spread of their scores (the
difference and its way to base 2 round, then the exponential, the sum and the quotient); bf16 roundings as in the step's
test."""
import pytest

from _helpers import say
from test_moe import block_inputs, rel

torch = pytest.importorskip("torch")
moe = pytest.importorskip("paper_2512_16512_amd.moe")

U = 2.0 ** -24


@pytest.fixture
def gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU visible")


def scores_of(T, E, dtype, seed=3):
    """No two of a row alike, so that there is one order of the choices."""
    g = torch.Generator().manual_seed(seed)
    if dtype == torch.bfloat16:
        s = torch.stack([torch.randperm(251, generator=g)[:E] for _ in range(T)]) / 32 - 4
    else:
        s = torch.randn(T, E, generator=g)
    s = s.to(dtype)
    assert all(len(set(row)) == E for row in s.tolist())
    return s


def reference(scores, top):
    """p of the rows sorted by expert, in 64 bits, differentiable."""
    v, e = torch.sort(scores, dim=1, descending=True)
    order = torch.sort(e[:, :top].flatten(), stable=True).indices
    return torch.softmax(v[:, :top], 1).flatten()[order]


# On the CPU: the routing of what is no plain tensor is torch's.


def test_fake_scores_are_routed_as_shapes():
    from torch._subclasses.fake_tensor import FakeTensorMode
    with FakeTensorMode():
        scores = torch.empty(8, 16, device="cuda:0")
        token, ends, p, which = moe.route(scores, 2)
        r = moe.routing(scores, 2)
    assert token.shape == p.shape == which.shape == (16,) and ends.shape == (16,) and ends.dtype == torch.int32
    assert r.expert.shape == r.row.shape == (8, 2) and r.counts.shape == (16,)


def test_symbols_and_compiled_programs_on_the_cpu():
    scores = scores_of(6, 9, torch.float32)
    want = moe.route(scores, 2)
    for name, f in (("symbols", torch.fx.symbolic_trace(lambda s: moe.route(s, 2))),
                    ("compiled", torch.compile(lambda s: moe.route(s, 2), backend="eager", fullgraph=True))):
        assert all(torch.equal(a, b) for a, b in zip(f(scores), want)), name


def test_gradient_of_the_weights_on_the_cpu():
    scores = scores_of(5, 7, torch.float64).requires_grad_()
    p = moe.route(scores, 3)[2]
    w = torch.linspace(1, 2, p.shape[0], dtype=p.dtype)
    (got,) = torch.autograd.grad((p * w).sum(), scores)
    leaf = scores.detach().clone().requires_grad_()
    (want,) = torch.autograd.grad((reference(leaf, 3) * w).sum(), leaf)
    assert torch.allclose(got, want, rtol=1e-5, atol=1e-7)


# On the GPU: whatever the type and size.


@pytest.mark.gpu
@pytest.mark.parametrize("T,E,top,dtype", [(40, 16, 2, torch.float32), (33, 60, 8, torch.float32), (1, 5, 5, torch.float32),
                                           (9, 1100, 3, torch.float32), (40, 16, 2, torch.bfloat16),
                                           (33, 200, 8, torch.bfloat16)])
def test_gradient_of_the_weights(gpu, T, E, top, dtype):
    scores = scores_of(T, E, dtype)
    leaf = scores.cuda().requires_grad_()
    say("route with a gradient", T, E, top, dtype)
    token, ends, p, which = moe.route(leaf, top)
    r = moe.routing(leaf, top)
    assert p.grad_fn is not None and r.p.grad_fn is not None
    w = torch.linspace(1, 2, p.shape[0], dtype=torch.float64)
    (got,) = torch.autograd.grad((p * w.cuda().float()).sum(), leaf)
    want_leaf = scores.double().requires_grad_()
    (want,) = torch.autograd.grad((reference(want_leaf, top) * w.float().double()).sum(), want_leaf)
    spread = 1 + (scores.double().amax(1, keepdim=True) - scores.double().amin(1, keepdim=True))
    tail = 2.0 ** -8 if dtype == torch.bfloat16 else U
    assert bool(((got.double().cpu() - want).abs() <= tail * want.abs() + 2 * 2 * (8 + top) * U * spread).all())
    with torch.no_grad():                     # nothing to follow: the operator's
        q = moe.routing(leaf, top)
    assert q.p.grad_fn is None and q.loss is not None if E <= moe.MOST_EXPERTS else q.loss is None
    assert torch.equal(q.expert, r.expert) and torch.equal(q.row, r.row) and torch.equal(q.token, r.token)
    assert torch.equal(q.ends, r.ends) and torch.equal(q.counts, r.counts)
    assert bool(((q.p - r.p).abs().double().cpu() <= 2 * 8 * U * spread).all())


@pytest.mark.gpu
@pytest.mark.parametrize("with_shared", [False, True])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_result_of_a_step_carries_its_routers_gradient(gpu, dtype, with_shared):
    norm, router, w1, w2, x, r, dout = block_inputs(moe, 120)
    router = router.to(dtype)
    shared = None
    if with_shared:
        g = torch.Generator().manual_seed(4)
        shared = tuple((0.1 * torch.randn(*s, generator=g)).to(t).cuda() for s, t in (
            ((256, 64), torch.bfloat16), ((64,), torch.float32), ((64, 256), torch.bfloat16), ((256,), torch.float32)))
    say("train step with a gradient", dtype, with_shared)
    plain = moe.train_step(x, r, norm, router, w1, w2, dout, shared=shared)
    leaf = router.clone().requires_grad_()
    got = moe.train_step(x, r, norm, leaf, w1, w2, dout, shared=shared)
    assert got[0].grad_fn is not None and plain[0].grad_fn is None
    assert rel(got[0].detach(), plain[0].double().cpu()) < 8 * 0.0017
    for a, b in zip(got[1:5], plain[1:5]):
        assert a.grad_fn is None and rel(a, b.double().cpu()) < 8 * 0.0017
    got[0].backward(dout.float())
    trained = moe.train_step(x, r, norm, leaf, w1, w2, dout, shared=shared, balance=0.0)
    assert trained.out.grad_fn is None and trained.drouter.grad_fn is None
    assert rel(leaf.grad, trained.drouter.double().cpu()) < 8 * 0.0017


@pytest.mark.gpu
def test_routing_is_traced_and_transformed(gpu):
    from torch.fx.experimental.proxy_tensor import make_fx
    first, other = scores_of(12, 9, torch.float32, 1).cuda(), scores_of(12, 9, torch.float32, 2).cuda()

    def weights(scores):
        return moe.route(scores, 3)[2]

    for name, traced in (("make_fx", make_fx(weights)(first)), ("jit", torch.jit.trace(weights, first, check_trace=False))):
        say("traced by", name)
        assert torch.allclose(traced(other), weights(other), rtol=1e-5)
    w = torch.linspace(1, 2, 36, device="cuda")
    say("transformed")
    got = torch.func.grad(lambda s: (weights(s) * w).sum())(first)
    leaf = first.clone().requires_grad_()
    (want,) = torch.autograd.grad((weights(leaf) * w).sum(), leaf)
    assert torch.allclose(got, want, rtol=1e-5, atol=1e-7)
    _, tangent = torch.func.jvp(weights, (first,), (other,))
    with torch.autograd.forward_ad.dual_level():
        dual = weights(torch.autograd.forward_ad.make_dual(first, other))
        assert torch.allclose(torch.autograd.forward_ad.unpack_dual(dual).tangent, tangent, rtol=1e-5, atol=1e-7)

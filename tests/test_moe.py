"""The mixture-of-experts block that runs the norm, 8-bit and grouped operators
together, against the same block in 64 bits.

Tolerances, as relative Frobenius errors: a value rounded to e4m3 is off by
2.6 % in the mean (3 bits after the point), and a served result passes four such
roundings (the normed rows, both weights, the hidden rows): 2 x 2.6 % x sqrt(4)
allows it twice that.  A value rounded to bfloat16 is off by 0.17 %; eight
roundings lie on the longest way of the training step."""
import pytest

from _helpers import say

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def moe():
    if not torch.cuda.is_available():
        pytest.skip("no GPU visible")
    from paper_2512_16512_amd import moe as mod
    return mod


def block(x, r, norm, w1, w2, token, ends, p, T, on=None):
    """The block in 64 bits for a given routing, differentiable.  ``on``: which hidden values the step had above zero
    (a value that rounding takes over zero turns its whole gradient on or off, which no tolerance on roundings
    describes); else those above zero in 64 bits."""
    h = x + r
    y = norm * h / torch.sqrt(h.square().mean(1, keepdim=True) + 1e-6)
    rows, parts, i = y[token], [], 0
    for e, j in enumerate(ends.tolist()):
        h = rows[i:j] @ w1[e]
        parts.append((torch.relu(h) if on is None else h * on[i:j]) @ w2[e])
        i = j
    return torch.zeros(T, x.shape[1], dtype=torch.float64).index_add(0, token, torch.cat(parts) * p[:, None])


def rel(got, want):
    return ((got.double().cpu() - want).norm() / want.norm()).item()


@pytest.mark.parametrize("tokens", [1, 7, 200])
def test_served_step(moe, tokens):
    D, F, E = 256, 384, 6
    norm, router, w1, w2 = moe.weights(E, D, F)
    g = torch.Generator().manual_seed(tokens)
    x, r = (torch.randn(tokens, D, generator=g).bfloat16().cuda() for _ in range(2))
    served = moe.Served(norm, router, w1, w2)
    say("served step", tokens)
    out, total = served.step(x, r)
    # the routing that the step took
    n = moe.rmsnorm(x, norm, r, quantize=True)
    token, ends, p, _ = moe.route(moe.matmul_fp8(n.out, n.scale, *served.router), 2)
    want = block(*(t.double().cpu() for t in (x, r, norm, w1, w2)), token.cpu(), ends.cpu(), p.double().cpu(), tokens)
    assert rel(out, want) < 4 * 0.026
    assert rel(total, (x.double() + r.double()).cpu()) < 2 ** -8


def test_train_step(moe):
    T, D, F, E = 300, 192, 320, 5
    norm, router, w1, w2 = moe.weights(E, D, F)
    g = torch.Generator().manual_seed(3)
    x, r, dout = (torch.randn(T, D, generator=g).bfloat16().cuda() for _ in range(3))
    say("train step")
    out, *grads = moe.train_step(x, r, norm, router, w1, w2, dout)
    n = moe.rmsnorm(x, norm, r)
    token, ends, p, _ = moe.route(n.out.float() @ router.float().t(), 2)
    on = (moe.matmul_grouped(n.out[token], w1, ends, relu=True, dtype=torch.bfloat16) > 0).double().cpu()
    leaf = [t.double().cpu().requires_grad_() for t in (x, norm, w1, w2)]
    want = block(leaf[0], r.double().cpu(), leaf[1], leaf[2], leaf[3], token.cpu(), ends.cpu(), p.double().cpu(), T, on)
    want.backward(dout.double().cpu())
    assert rel(out, want.detach()) < 8 * 0.0017
    for name, got, t in zip(("x", "norm", "w1", "w2"), grads, leaf):
        assert rel(got, t.grad) < 8 * 0.0017, name


def block_inputs(moe, T, D=256, F=384, E=6):
    norm, router, w1, w2 = moe.weights(E, D, F)
    g = torch.Generator().manual_seed(11)
    x, r, dout = (torch.randn(T, D, generator=g).bfloat16().cuda() for _ in range(3))
    return norm, router, w1, w2, x, r, dout


def test_steps_do_not_wait_for_the_gpu(moe):
    """The groups' ends stay on the device: nothing of a step is read back to the host."""
    norm, router, w1, w2, x, r, dout = block_inputs(moe, 200)
    served = moe.Served(norm, router, w1, w2)
    torch.cuda.synchronize()
    torch.cuda.set_sync_debug_mode("error")
    try:
        served.step(x, r)
        moe.train_step(x, r, norm, router, w1, w2, dout)
    finally:
        torch.cuda.set_sync_debug_mode("default")


def test_route_sorts_rows_by_expert(moe):
    """Also where experts at either end or in between get no row."""
    scores = torch.full((5, 7), -9.0)
    scores[:, [1, 4]] = torch.tensor([[3.0, 1], [0, 2], [5, 4], [1, 1.5], [2, 6]])
    token, ends, p, which = moe.route(scores.cuda(), 2)
    assert ends.dtype == torch.int32 and ends.tolist() == [0, 5, 5, 5, 10, 10, 10]
    assert token.tolist() == [0, 1, 2, 3, 4] * 2 and sorted(which.tolist()) == list(range(10))
    want = torch.softmax(scores[:, [1, 4]].double(), 1).t().flatten()
    assert torch.allclose(p.cpu().double(), want, rtol=1e-6, atol=0)
    _, ends, _, _ = moe.route(scores[:0].cuda(), 2)
    assert ends.tolist() == [0] * 7


def test_steps_give_the_same_bits_again(moe):
    """A token's experts are summed in their order, however many it has."""
    norm, router, w1, w2, x, r, dout = block_inputs(moe, 3000, 512, 128, 16)
    served = moe.Served(norm, router, w1, w2, top=8)
    first = served.step(x, r)
    train = moe.train_step(x, r, norm, router, w1, w2, dout, top=8)
    for _ in range(4):
        assert all(torch.equal(a, b) for a, b in zip(first, served.step(x, r)))
        assert all(torch.equal(a, b) for a, b in zip(train, moe.train_step(x, r, norm, router, w1, w2, dout, top=8)))


def test_steps_of_no_tokens(moe):
    norm, router, w1, w2, x, r, dout = block_inputs(moe, 0)
    out, total = moe.Served(norm, router, w1, w2).step(x, r)
    assert out.shape == total.shape == (0, 256) and out.dtype == torch.float32
    out, dx, dnorm, dw1, dw2 = moe.train_step(x, r, norm, router, w1, w2, dout)
    assert out.shape == dx.shape == (0, 256) and dw1.shape == w1.shape and dw2.shape == w2.shape
    assert not any(bool(t.any()) for t in (dnorm, dw1, dw2))

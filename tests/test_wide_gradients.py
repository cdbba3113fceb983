"""Gradients of rows so wide that the launch over their columns would have 2^32 threads or more: columns on both sides of
where the launches part, and the last, against sums in 64 bits (n fp32 terms are within n 2^-24 of their magnitudes' sum,
the products round once more)."""
import pytest

from _helpers import say

torch = pytest.importorskip("torch")
x = pytest.importorskip("paper_2512_16512_amd")

pytestmark = pytest.mark.gpu

U = 2.0 ** -24


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU visible")
    yield
    torch.cuda.empty_cache()


def filled(rows, D, seed):
    t = torch.empty(rows, D, dtype=torch.bfloat16, device="cuda")
    return t.normal_(generator=torch.Generator(device="cuda").manual_seed(seed))


def around(D):
    at = torch.cat([torch.arange(i, i + 40) for i in (0, D // 2, D - 40)] + [torch.arange(max(0, 2 ** b - 20), 2 ** b + 20) for b in (24, 25)])
    return at[at < D].cuda()


def test_layernorm_gradient():
    T, D = 257, 2 ** 25 + 24
    rows, dy = filled(T, D, 1), filled(T, D, 2)
    mean, rstd = torch.zeros(T, device="cuda"), torch.ones(T, device="cuda")
    say("layernorm_backward", T, D)
    dx, dw, db = x.layernorm_backward(dy, rows, torch.ones(D, dtype=torch.bfloat16, device="cuda"), mean, rstd)
    del dx
    c = around(D)
    d, h = dy[:, c].double(), rows[:, c].double()
    assert bool(((db[c].double() - d.sum(0)).abs() <= T * U * d.abs().sum(0)).all())
    assert bool(((dw[c].double() - (d * h).sum(0)).abs() <= (T + 2) * U * (d * h).abs().sum(0)).all())


def test_gradients_of_no_rows():
    D = 2 ** 26 + 8
    for f, n in ((x.layernorm_backward, 2), (x.rmsnorm_backward, 1)):
        dirty = torch.full((2, D), float("nan"), device="cuda")
        del dirty                              # (what the results' memory held)
        none, w = torch.empty(0, D, device="cuda"), torch.ones(D, device="cuda")
        stats = [torch.empty(0, device="cuda")] * n
        say("no rows", f.__name__)
        for g in f(none, none, w, *stats)[1:]:
            assert g.shape == (D,) and not bool(g.any())


def test_activation_gradient():
    N = 2 ** 30                                # the widest row there may be
    z, dy = filled(1, N, 3), filled(1, N, 4)
    say("activation_backward", N)
    dz, db = x.activation_backward(dy, z, "relu")
    want = dy.float() * (z > 0)
    assert torch.equal(db, want[0]) and torch.equal(dz, want.bfloat16())

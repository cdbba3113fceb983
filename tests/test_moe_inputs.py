"""Layouts in which a mixture-of-experts step takes its router, its scores and its output's gradient: the same bits as of
contiguous copies, but of rows that begin off 16 bytes, which the linear layer sums in another order: fp32 sums that differ by
2 u a term, u = 2^-24, and here and there round to the other bf16 neighbour, within what the step's test allows."""
import pytest

from _helpers import say
from test_moe import block_inputs, rel

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def moe():
    if not torch.cuda.is_available():
        pytest.skip("no GPU visible")
    from paper_2512_16512_amd import moe as mod
    return mod


@pytest.mark.parametrize("balance", [None, 0.5])
def test_train_step_of_views(moe, balance):
    norm, router, w1, w2, x, r, _ = block_inputs(moe, 100)
    row = torch.randn(256, generator=torch.Generator().manual_seed(1)).cuda()
    wide = torch.zeros(6, 300, dtype=torch.bfloat16, device="cuda")
    wide[:, 3:259] = router
    routers = {"a transposed view": router.t().contiguous().t(), "part of a wider matrix": wide[:, 3:259]}
    douts = {"one row for all, bf16": row.bfloat16().expand(100, 256), "one row for all, fp32": row.expand(100, 256),
             "one value for all": row[:1].expand(100, 256), "64 bits": row.double().expand(100, 256),
             "a transposed view": row.expand(100, 256).t().contiguous().t()}

    def step(router, dout):
        got = moe.train_step(x, r, norm, router, w1, w2, dout, balance=balance)
        return [t for t in got if t is not None]

    want = step(router, row.expand(100, 256).contiguous())
    for name, view in routers.items():
        say("router", name, balance)
        assert torch.equal(view, router)
        got = step(view, douts["one row for all, fp32"])
        if view.data_ptr() % 16 or view.stride(0) % 8:
            assert all(rel(a, b.double().cpu()) < 8 * 0.0017 for a, b in zip(got, want)), name
        else:
            assert all(torch.equal(a, b) for a, b in zip(got, want)), name
    for name, dout in douts.items():
        say("dout", name, balance)
        got = step(router, dout)
        assert all(torch.equal(a, b) for a, b in zip(got, step(router, dout.to(
            torch.float32 if dout.dtype == torch.float64 else dout.dtype).contiguous()))), name


def test_route_of_rows_that_share_memory(moe):
    scores = torch.randn(40, generator=torch.Generator().manual_seed(2)).cuda()
    for view in (scores.expand(30, 40), scores.bfloat16().expand(30, 40), scores.as_strided((10, 16), (2, 1))):
        say("route", view.dtype, view.stride())
        for got, want in zip(moe.route(view, 3), moe.route(view.contiguous(), 3)):
            assert torch.allclose(got.double(), want.double(), rtol=1e-6, atol=0)      # (one path may be torch's)

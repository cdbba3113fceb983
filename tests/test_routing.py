"""The router of a mixture of experts and the sum of its experts' rows, with their
gradients, against their definitions in 64 bits and, for places and counts, exactly.

Tolerances.  u = 2^-24 is half a unit in the last place of fp32; 2^(v log2 e) is within
2u |v| (the product and its constant) and 2u (the instruction) of e^v; a sum of n terms is within
n u of the sum of their magnitudes, those over a row's E scores within (E / 16 + 6) u (lanes of at most
16 neighbours each, joined by halves).  Rounding to bf16 is within 2^-8 of the value."""
import math

import numpy as np
import pytest

from _helpers import say
from test_operators import BF16, U, as_type, dev, host, normal, within

torch = pytest.importorskip("torch")
x = pytest.importorskip("paper_2512_16512_amd")


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU visible")


pytestmark = pytest.mark.gpu


def chosen_of(scores, top):
    """[T, top]: by score, a NaN above every number; of equal ones the lowest index."""
    out = np.zeros((scores.shape[0], top), dtype=np.int64)
    for t, row in enumerate(scores.double().tolist()):
        rank = sorted(range(len(row)), key=lambda e: (0, 0.0, e) if math.isnan(row[e]) else (1, -row[e], e))
        out[t] = rank[:top]
    return out


def softmax(v):
    """In 64 bits; zeros where every value is -inf, NaN with a NaN or an infinity above."""
    top = v.amax(-1, keepdim=True)
    q = torch.exp(v - top)
    return torch.where(torch.isneginf(top), torch.zeros_like(v), q / q.sum(-1, keepdim=True))


def softmax_bound(v):
    """Relative, of values up to `spread` below the largest."""
    fine = torch.where(torch.isfinite(v), v, torch.zeros_like(v))
    spread = fine.amax(-1, keepdim=True) - fine
    n = v.shape[-1] / 16 + 6
    # e^(v - top) (the difference rounds too), and the largest such error once more in the sum
    return (4 * spread + 2 + n + 6) * U + 8 * U * spread.clamp_max(30).amax(-1, keepdim=True)


def check_routing(r, scores, top, mask, what):
    T, E = scores.shape
    there = np.ones(T, bool) if mask is None else mask.numpy()
    want = chosen_of(scores, top)
    expert = np.where(there[:, None], want, -1)
    assert r.expert.dtype == r.row.dtype == r.token.dtype == r.counts.dtype == r.ends.dtype == torch.int32
    assert r.p.dtype == r.loss.dtype == torch.float32 and r.loss.shape == ()
    assert np.array_equal(r.expert.cpu().numpy(), expert), what
    counts = np.bincount(expert[expert >= 0], minlength=E)[:E]
    assert np.array_equal(r.counts.cpu().numpy(), counts) and np.array_equal(r.ends.cpu().numpy(), np.cumsum(counts)), what
    # rows: by expert, then by token
    pairs = sorted((e, t, j) for t in range(T) for j, e in enumerate(expert[t]) if e >= 0)
    row, token = np.full((T, top), -1), np.full(T * top, -1)
    for i, (_, t, j) in enumerate(pairs):
        row[t, j], token[i] = i, t
    assert np.array_equal(r.row.cpu().numpy(), row), what
    assert np.array_equal(r.token.cpu().numpy(), token), what
    v = scores.double()
    picked = torch.gather(v, 1, torch.from_numpy(want))
    p = torch.where(torch.from_numpy(there)[:, None], softmax(picked), torch.zeros(()).double())
    within(host(r.p), p, torch.nan_to_num(p * softmax_bound(picked)) + 2.0 ** -126, what + " p")
    q = softmax(v)[torch.from_numpy(there)]
    n = max(int(there.sum()), 1)
    c = torch.from_numpy(counts).double()
    loss = E / (top * n * n) * (c * q.sum(0)).sum()
    off = E / (top * n * n) * (c * (q * torch.nan_to_num(softmax_bound(v[torch.from_numpy(there)]))).sum(0)).sum()
    within(host(r.loss), loss, torch.nan_to_num(off + (T + E + 8) * U * loss.abs()), what + " loss")


SIZES = [(1, 1, 1), (1, 64, 8), (2, 7, 7), (5, 16, 2), (63, 8, 2), (64, 64, 6), (65, 33, 4), (130, 60, 6), (1000, 128, 8),
         (257, 256, 8), (70, 200, 16), (3, 257, 8), (300, 1024, 16), (200, 600, 3), (4097, 16, 1), (16, 300, 4),
         (17, 20, 2), (2100, 400, 4), (2049, 1000, 2), (9000, 40, 2), (16700, 12, 2)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T,E,top", SIZES)
def test_route_experts(T, E, top, dtype):
    for masked in (False, True):
        scores = as_type(normal(T + E, T, E) + 0.8 * normal(E, E), dtype)        # (bf16: with ties)
        mask = torch.from_numpy(np.random.RandomState(T).rand(T) < 0.7) if masked else None
        for odd in (False, True):
            what = "route_experts %s" % ((T, E, top, dtype, masked, odd),)
            say(what)
            r = x.route_experts(dev(scores, odd), top, None if mask is None else mask.cuda())
            check_routing(r, scores, top, mask, what)


def test_route_experts_of_many_tokens():
    """Workgroups of several groups of tokens, the last one short."""
    T, E, top = 33000, 24, 3
    scores = as_type(normal(1, T, E), "bf16")
    mask = torch.from_numpy(np.random.RandomState(2).rand(T) < 0.9)
    say("route_experts", T, E, top)
    check_routing(x.route_experts(dev(scores), top, mask.cuda()), scores, top, mask, "many")


def test_route_experts_ties_and_special_scores():
    inf, nan = float("inf"), float("nan")
    scores = torch.tensor([[1.0, 1, 1, 1, 1], [0.0, -0.0, 0.0, -0.0, -1], [-inf, 2, -inf, 1, -inf], [-inf] * 5,
                           [1, nan, 3, nan, 2], [5, -inf, -inf, -inf, -inf], [3e38, -3e38, 0, 1e-40, -1e-40],
                           [1, 2, inf, 0, 0], [-nan, 1, 2, 3, 4]])
    for top in (1, 2, 3, 5):
        say("special scores", top)
        r = x.route_experts(dev(scores), top)
        assert np.array_equal(r.expert.cpu().numpy(), chosen_of(scores, top))
        p = host(r.p)
        assert bool(torch.isnan(p[[4, 7, 8]]).any(1).all()) and not bool(torch.isnan(p[[0, 1, 2, 3, 5, 6]]).any())
        assert bool((p[3] == 0).all()) and p[5, 0] == 1 and bool((p[5, 1:] == 0).all())
        assert bool(torch.isnan(r.loss.cpu()))
    fine = scores[[0, 1, 2, 3, 5, 6]]
    check_routing(x.route_experts(dev(fine), 2), fine, 2, None, "finite ones")


@pytest.mark.parametrize("T", [0, 5, 300])
def test_route_experts_without_tokens(T):
    mask = torch.zeros(T, dtype=torch.bool, device="cuda")
    r = x.route_experts(torch.randn(T, 12, device="cuda"), 4, mask)
    assert r.expert.shape == (T, 4) and bool((r.expert == -1).all()) and bool((r.row == -1).all())
    assert bool((r.token == -1).all()) and not bool(r.counts.any()) and not bool(r.ends.any())
    assert not bool(r.p.any()) and r.loss.item() == 0
    ds = x.route_experts_backward(torch.randn(T, 4, device="cuda"), torch.randn(T, 12, device="cuda"), r.expert, r.p,
                                  r.counts, 0.5)
    assert ds.shape == (T, 12) and not bool(ds.any())


def test_balance_loss_of_equal_and_of_one_sided_routing():
    E = 8
    even = torch.zeros(E * 4, E)
    even[torch.arange(E * 4), torch.arange(E * 4) % E] = 1.0
    assert abs(x.route_experts(dev(even), 1).loss.item() - 1) < 1e-5
    one = torch.zeros(50, E)
    one[:, 3] = 40.0
    assert abs(x.route_experts(dev(one), 1).loss.item() - E) < 1e-5


def scores_gradient(scores, top, there, dp, dloss):
    """ds in 64 bits, and the magnitudes that its error scales with."""
    v, E = scores.double(), scores.shape[1]
    expert = torch.from_numpy(chosen_of(scores, top))
    picked = torch.gather(v, 1, expert)
    p, q = softmax(picked) * there[:, None], softmax(v) * there[:, None]
    n = max(int(there.sum()), 1)
    c = torch.bincount(expert[there].flatten(), minlength=E).double()
    scale = dloss * E / (top * n * n)
    one = scale * q * (c - (q * c).sum(1, keepdim=True))
    two = p * (dp.double() - (p * dp.double()).sum(1, keepdim=True))
    mag = abs(scale) * q * (c + (q * c).sum(1, keepdim=True))
    mag2 = p * (dp.double().abs() + (p * dp.double().abs()).sum(1, keepdim=True))
    return one.scatter_add(1, expert, two), mag.scatter_add(1, expert, mag2), expert, p, c


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T,E,top", [(1, 1, 1), (1, 64, 8), (5, 16, 2), (65, 33, 4), (130, 60, 6), (1000, 128, 8),
                                     (70, 200, 16), (300, 1024, 16), (40000, 7, 2)])
def test_route_experts_backward(T, E, top, dtype):
    scores = as_type(normal(T + E, T, E) + 0.8 * normal(E, E), dtype)
    dp = normal(3, T, top).float()
    for masked in (False, True):
        there = torch.from_numpy(np.random.RandomState(T).rand(T) < 0.7) if masked else torch.ones(T, dtype=torch.bool)
        mask = there.cuda() if masked else None
        for odd in (False, True):
            say("route_experts_backward", T, E, top, dtype, masked, odd)
            ref, mag, expert, p, c = scores_gradient(scores, top, there, dp, 0.3)
            r = x.route_experts(dev(scores, odd), top, mask)
            ds = x.route_experts_backward(dev(dp), dev(scores, odd), r.expert, r.p, r.counts, 0.3)
            assert ds.dtype == scores.dtype
            tail = BF16 if dtype == "bf16" else U
            # p and q once each, with their sums, and p as the forward pass rounded it
            rel = (3 * softmax_bound(scores.double()) + (E + 16) * U).amax()
            within(host(ds), ref, tail * ref.abs() + 2 * rel * mag + 2.0 ** -126, "ds")
            other = torch.float32 if dtype == "bf16" else torch.bfloat16
            got = x.route_experts_backward(None, dev(scores, odd), r.expert, r.p, r.counts, 0.3, dtype=other)
            ref, mag, *_ = scores_gradient(scores, top, there, torch.zeros_like(dp), 0.3)
            assert got.dtype == other
            within(host(got), ref, BF16 * ref.abs() + 2 * rel * mag + 2.0 ** -126, "balance alone")


def test_route_experts_backward_against_differences():
    """Central differences of loss * 0.7 + <p, dp> with the choice as it is (no step changes it)."""
    T, E, top, step = 40, 24, 4, 1e-6
    scores, dp = normal(1, T, E).float(), normal(2, T, top).float()
    r = x.route_experts(dev(scores), top)
    ds = host(x.route_experts_backward(dev(dp), dev(scores), r.expert, r.p, r.counts, 0.7))
    expert, c = r.expert.cpu().long(), r.counts.cpu().double()

    def value(v):
        loss = E / (top * T * T) * (c * softmax(v).sum(0)).sum()
        return 0.7 * loss + (softmax(torch.gather(v, 1, expert)) * dp.double()).sum()

    for seed in range(4):
        d = normal(10 + seed, T, E)
        num = (value(scores.double() + step * d) - value(scores.double() - step * d)) / (2 * step)
        assert abs(num.item() - (ds * d).sum().item()) <= 1e-5 * ds.norm().item() * d.norm().item()


# ---------------------------------------------------------------- combine


def routing(T, top, seed, masked=True):
    """row, token and p of a random routing of T tokens, a fifth of them masked, the rows in any order."""
    g = np.random.RandomState(seed)
    there = g.rand(T) < (0.8 if masked else 2)
    n = int(there.sum()) * top
    row, token = np.full((T, top), -1, np.int32), np.full(T * top, -1, np.int32)
    row[there] = g.permutation(n).reshape(-1, top)
    token[row[there].reshape(-1)] = np.repeat(np.nonzero(there)[0], top)
    return torch.from_numpy(row), torch.from_numpy(token), torch.softmax(normal(seed, T, top), 1).float()


COMBINE = [(0, 2, 8), (1, 1, 1), (1, 8, 2048), (3, 2, 7), (5, 6, 513), (33, 16, 128), (100, 3, 1021), (257, 8, 512),
           (20, 9, 4096), (40, 17, 40)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T,top,D", COMBINE)
def test_combine_experts(T, top, D, dtype):
    row, _, p = routing(T, top, T + D)
    rows, res = as_type(normal(D, T * top, D), dtype), normal(T, T, D)
    g = torch.where(row[:, :, None] >= 0, rows.double()[row.long().clamp_min(0)] if T else torch.zeros(0, top, D).double(), 0.0)
    for weights in (p, None):
        w = torch.ones(T, top).double() if weights is None else weights.double()
        for r_t, out in ((None, "f32"), ("f32", "bf16"), ("bf16", "f32")):
            r = None if r_t is None else as_type(res, r_t)
            ref = (w[:, :, None] * g).sum(1) + (0 if r is None else r.double())
            mag = (w[:, :, None] * g.abs()).sum(1) + (0 if r is None else r.double().abs())
            tail = BF16 if out == "bf16" else U
            for odd in (False, True):
                say("combine_experts", T, top, D, dtype, r_t, out, odd)
                got = x.combine_experts(dev(rows, odd), dev(row), None if weights is None else dev(weights),
                                        None if r is None else dev(r, odd), torch.bfloat16 if out == "bf16" else None)
                assert got.dtype == (torch.bfloat16 if out == "bf16" else torch.float32)
                within(host(got), ref, tail * ref.abs() + (1 + tail) * (top + 2) * U * mag, "combine")


def test_combine_experts_does_not_read_what_no_token_has():
    """NaN in the rows behind the last one, in those of masked choices, and places outside the array."""
    T, top, D = 50, 3, 200
    row, token, p = routing(T, top, 7)
    rows = normal(1, T * top, D).float()
    want = host(x.combine_experts(dev(rows), dev(row), dev(p)))
    dout = normal(2, T, D).float()
    drows, dp = x.combine_experts_backward(dev(dout), dev(rows), dev(row), dev(token), dev(p))
    rows[token < 0] = float("nan")
    masked = row[:, 0] < 0
    far = row.clone()
    far[masked] = torch.tensor([-1, 2 ** 31 - 1, T * top], dtype=torch.int32)
    p[masked] = float("nan")
    assert torch.equal(host(x.combine_experts(dev(rows), dev(far), dev(p))), want)
    again = x.combine_experts_backward(dev(dout), dev(rows), dev(far), dev(token), dev(p))
    assert torch.equal(again[0], drows) and torch.equal(again[1], dp)
    assert not bool(drows[dev(token) < 0].any()) and not bool(dp[dev(masked)].any())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T,top,D", COMBINE)
def test_combine_experts_backward(T, top, D, dtype):
    row, token, p = routing(T, top, T + D)
    rows = as_type(normal(D, T * top, D), dtype)
    tail = BF16 if dtype == "bf16" else U
    for g_t in ("f32", "bf16"):
        dout = as_type(normal(T, T, D), g_t)
        drows, dp, mag = torch.zeros(T * top, D).double(), torch.zeros(T, top).double(), torch.zeros(T, top).double()
        for j in range(top):
            at = row[:, j] >= 0
            i = row[at, j].long()
            drows[i] = p.double()[at, j:j + 1] * dout.double()[at]
            dp[at, j] = (rows.double()[i] * dout.double()[at]).sum(1)
            mag[at, j] = (rows.double()[i] * dout.double()[at]).abs().sum(1)
        for odd in (False, True):
            say("combine_experts_backward", T, top, D, dtype, g_t, odd)
            got, gp = x.combine_experts_backward(dev(dout, odd), dev(rows, odd), dev(row), dev(token), dev(p))
            assert got.dtype == rows.dtype and gp.dtype == torch.float32
            within(host(got), drows, (tail + 2 * U) * drows.abs(), "drows")
            within(host(gp), dp, (D + 8) * U * mag, "dp")


def test_combine_experts_gradients_against_differences():
    T, top, D, step = 12, 3, 70, 1e-6
    row, token, p = routing(T, top, 3)
    rows, dout = normal(1, T * top, D).float(), normal(2, T, D).float()
    drows, dp = (host(t) for t in x.combine_experts_backward(dev(dout), dev(rows), dev(row), dev(token), dev(p)))

    def value(a, w):
        return (torch.where(row[:, :, None] >= 0, a[row.long().clamp_min(0)], 0.0) * w[:, :, None] * dout.double()[:, None]).sum()

    a, w = rows.double(), p.double()
    for seed in range(3):
        u, v = normal(20 + seed, T * top, D), normal(30 + seed, T, top)
        num = (value(a + step * u, w) - value(a - step * u, w)) / (2 * step)
        assert abs(num.item() - (drows * u).sum().item()) <= 1e-5 * drows.norm().item() * u.norm().item()
        num = (value(a, w + step * v) - value(a, w - step * v)) / (2 * step)
        assert abs(num.item() - (dp * v).sum().item()) <= 1e-5 * dp.norm().item() * v.norm().item()

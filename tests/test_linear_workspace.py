"""The linear layer's workspace has an upper bound, whatever its operands (host only)."""
import math
import random

import pytest

x = pytest.importorskip("paper_2512_16512_amd")

AT = 0x10000               # an address at 16 bytes, never read
MOST, COPIES = 640 << 20, 512 << 20


def workspaces(T, N, K, off=0, pad=0):
    """Of the layer in both layouts and of its weights' gradient: operands `off` elements behind 16 bytes, rows `pad` longer."""
    a, b = AT + 2 * off, AT + 2 * off
    return (x.xtc_linear_workspace(T, N, K, a, K + pad, b, N + pad, 0), x.xtc_linear_workspace(T, N, K, a, K + pad, b, K + pad, 1),
            x.xtc_linear_wgrad_workspace(T, N, K, a, K + pad, b, N + pad))


@pytest.mark.parametrize("T,N,K", [(600000, 1024, 4097), (1000000, 4096, 4095), (300000, 4096, 8193), (1 << 26, 8, 9),
                                   (70000, 4096, 4097), (5, 300001, 8193), (4096, 4097, 300001), (0x7FFFFF00, 1, 1),
                                   (0x7FFFFF00, 0x7FFFFF00, 0x7FFFFF00), (0x7FFFFEFF, 0x7FFFFEFF, 0x7FFFFEFF)])
def test_large_operands_at_odd_widths(T, N, K):
    assert all(0 <= w <= MOST for w in workspaces(T, N, K))


def test_operands_are_still_copied_where_that_is_little():
    """12190 rows, 803 x 6111: both copies are 184 MB and take a third off the gradient's time."""
    assert workspaces(12190, 6111, 803)[2] >= 12190 * (808 + 6112) * 2


def test_many_sizes():
    rng = random.Random(5)

    def log(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    seen = 0
    for _ in range(20000):
        T, N, K = log(1, 1 << 23), log(1, 1 << 16), log(1, 1 << 16)
        if rng.random() < 0.2:
            T, N, K = log(1, 1 << 12), log(1, 1 << 12), log(1, 1 << 25)
        off = rng.randrange(8)
        both = workspaces(T, N, K, off) if rng.random() < 0.5 else workspaces(T, N, -(-K // 8) * 8, 0, 8)
        assert all(0 <= w <= MOST for w in both), (T, N, K, off, both)
        seen += any(w > 0 for w in both)
    assert seen > 1000


@pytest.mark.gpu
def test_operands_past_the_bound_are_right():
    """573 MB of rows off 16 bytes, which no workspace holds: a layer and its weights' gradient by rows at any address.  A sum
    of n products is within 2u n of the sum of their magnitudes (u = 2^-24, the matrix cores may truncate)."""
    torch = pytest.importorskip("torch")
    if not torch.cuda.is_available():
        pytest.skip("no GPU visible")
    from _helpers import say
    T, K, N, u = 70000, 4097, 72, 2.0 ** -24
    g = torch.Generator(device="cuda").manual_seed(2)
    a = torch.randn(T, K, device="cuda", generator=g).bfloat16()
    b = (torch.randn(K, N, device="cuda", generator=g) / 64).bfloat16()
    dy = torch.randn(T, N, device="cuda", generator=g).bfloat16()
    assert workspaces(T, N, K)[0] < COPIES and x.xtc_linear_wgrad_workspace(T, N, K, AT, K, AT, N) < COPIES
    rows = torch.cat([torch.arange(i, min(i + 70, T)) for i in (0, 32700, 65500, T - 70)]).cuda()
    say("linear past the bound")
    got = x.linear(a, b).double()[rows]
    some = a[rows].double()
    assert bool(((got - some @ b.double()).abs() <= 2 * u * (K + 24) * (some.abs() @ b.double().abs())).all())
    say("linear_wgrad past the bound")
    got = x.linear_wgrad(a, dy).double()[-70:]
    some = a[:, -70:].double().t().contiguous()
    assert bool(((got - some @ dy.double()).abs() <= 2 * u * (T + 24) * (some.abs() @ dy.double().abs())).all())

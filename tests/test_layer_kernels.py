"""Every kernel, with and without splits, among which a linear layer chooses, at a size that takes it.  On the CPU: the
sizes below reach all of them, by the library's own choice.  On the GPU: each against the definition in 64 bits,
within the bounds of test_layer_operators.py."""
import ctypes

import pytest

from _helpers import say

torch = pytest.importorskip("torch")
x = pytest.importorskip("paper_2512_16512_amd")

from test_operators import BF16, U, as_type, normal  # noqa: E402

LAYER, TURNED, WGRAD = 1, 2, 3      # as the library numbers them

# kind, elements that rows begin behind 16 bytes, rows, N, K
SIZES = [
    (1, 0, 8274, 904, 72), (1, 0, 8801, 416, 264), (1, 0, 8462, 72, 3360), (1, 0, 8212, 400, 72),
    (1, 0, 8668, 72, 2640), (1, 0, 8408, 200, 72), (1, 0, 4270, 72, 3568), (1, 0, 8313, 72, 264),
    (1, 0, 5655, 72, 72), (1, 0, 3, 72, 72), (1, 0, 3, 4104, 72), (1, 0, 3, 1912, 4024), (1, 0, 17, 4152, 72),
    (1, 0, 17, 1176, 4120), (1, 0, 2732, 72, 72), (1, 0, 37, 1208, 4192), (1, 0, 4115, 72, 72),
    (1, 0, 50, 3864, 3976), (1, 1, 65, 2856, 72), (1, 1, 3, 4184, 800), (1, 1, 3, 72, 72), (1, 1, 3, 483, 4176),
    (1, 1, 8237, 904, 72), (1, 1, 1243, 3259, 264), (1, 1, 1753, 3507, 72), (1, 1, 5499, 531, 72),
    (1, 1, 589, 867, 4136), (1, 1, 1256, 787, 1392), (1, 1, 3470, 528, 949), (1, 1, 3, 72, 197), (1, 1, 3, 4107, 688),
    (1, 1, 1417, 72, 456), (1, 1, 300, 816, 616), (1, 1, 1085, 467, 968), (2, 0, 8255, 912, 72),
    (2, 0, 1181, 3416, 200), (2, 0, 8405, 72, 3424), (2, 0, 8480, 392, 72), (2, 0, 8395, 200, 72),
    (2, 0, 4402, 72, 3288), (2, 0, 8203, 72, 392), (2, 0, 2955, 72, 4008), (2, 0, 4105, 72, 72),
    (2, 0, 2602, 136, 4056), (2, 0, 3, 72, 72), (2, 0, 3, 4160, 216), (2, 0, 18, 4128, 72), (2, 0, 36, 4144, 72),
    (2, 0, 4118, 72, 1056), (2, 1, 3, 72, 72), (2, 1, 3, 3011, 1312), (2, 1, 3, 72, 133), (2, 1, 3, 728, 4165),
    (2, 1, 8409, 899, 72), (2, 1, 1137, 3672, 200), (2, 1, 1668, 3016, 72), (2, 1, 7182, 387, 72),
    (2, 1, 841, 616, 4112), (2, 1, 808, 1267, 1816), (2, 1, 2337, 1696, 261), (2, 1, 3, 72, 453),
    (2, 1, 18, 2360, 784), (2, 1, 904, 131, 736), (2, 1, 293, 936, 1608), (2, 1, 550, 899, 2677),
    (3, 0, 3, 2064, 3880), (3, 0, 332, 1208, 3272), (3, 0, 6662, 1176, 136), (3, 0, 3, 72, 72), (3, 0, 577, 72, 72),
    (3, 1, 3, 72, 72), (3, 1, 581, 72, 72), (3, 1, 513, 72, 72), (3, 1, 1295, 136, 2173), (3, 1, 3, 2659, 3464),
    (3, 1, 385, 2251, 1997), (3, 1, 3, 2699, 2261),
]


@pytest.fixture(scope="module")
def place():
    f = ctypes.CDLL(x.LIB_PATH).xtc_test_linear_kernel
    f.argtypes = [ctypes.c_int32] + [ctypes.c_int64] * 3 + [ctypes.c_int32] + [ctypes.POINTER(ctypes.c_int32)] * 2

    def at(kind, off, T, N, K):
        n, splits = ctypes.c_int32(), ctypes.c_int32()
        p = f(kind, T, N, K, off, ctypes.byref(n), ctypes.byref(splits))
        return p, n.value, splits.value

    return at


@pytest.mark.parametrize("off", [0, 1])
@pytest.mark.parametrize("kind", [LAYER, TURNED, WGRAD])
def test_the_sizes_reach_every_kernel(place, kind, off):
    seen = [place(*size) for size in SIZES if size[:2] == (kind, off)]
    assert {p for p, _, _ in seen} == set(range(seen[0][1]))
    assert any(splits > 1 for _, _, splits in seen) and any(splits == 1 for _, _, splits in seen)


def inside(t, off):
    """On the GPU, its rows ``off`` elements behind 16 bytes where its own width is a multiple of them."""
    wide = torch.full((t.shape[0], t.shape[1] + (-t.shape[1] % 8 if off == 0 else 0) + 8 * off), float("nan"), dtype=t.dtype)
    wide[:, off:off + t.shape[1]] = t
    return wide.cuda()[:, off:off + t.shape[1]]


@pytest.mark.gpu
@pytest.mark.parametrize("kind,off,T,N,K", SIZES)
def test_every_kernel(kind, off, T, N, K):
    if not torch.cuda.is_available():
        pytest.skip("no GPU visible")
    a = as_type(normal(T + K, T, K), "bf16")
    b = as_type(normal(N, T, N) if kind == WGRAD else normal(N, K, N) / K ** 0.5, "bf16")
    p, q = a.cuda().double(), b.cuda().double()
    if kind == WGRAD:
        p = p.t().contiguous()
    ref, mag, n = p @ q, p.abs() @ q.abs(), p.shape[1]
    bias, res = normal(1, N).float().cuda(), as_type(normal(2, T, N), "bf16").cuda()
    stored = inside(b.t().contiguous() if kind == TURNED else b, off)
    a = inside(a, off)
    for out in (torch.float32, torch.bfloat16):
        say("every kernel", kind, off, T, N, K, out)
        tail = BF16 if out == torch.bfloat16 else U
        e = 2 * U * (n + 24) * mag
        if kind == WGRAD:
            got, want = x.linear_wgrad(a, stored, dtype=out), ref
        else:
            got, z = x.linear(a, stored, bias, res, "relu", kind == TURNED, True, dtype=out)
            want = ref + bias.double()
            e = e + 2 * U * (want.abs() + bias.double().abs())
            assert bool(((z.double() - want).abs() <= tail * want.abs() + (1 + tail) * e).all())
            want = want.clamp_min(0) + res.double()
            e = e + 2 * U * (want.abs() + res.double().abs())
        assert got.dtype == out and got.shape == want.shape
        assert bool(((got.double() - want).abs() <= tail * want.abs() + (1 + tail) * e).all())

"""Every kernel among which the 8-bit and grouped products choose, at a size that
takes it.  On the CPU: the sizes below reach all of them, by the library's own choice.
On the GPU: each against the definition in 64 bits, within the bounds of
test_operators.py."""
import ctypes

import numpy as np
import pytest

from _helpers import say

torch = pytest.importorskip("torch")
x = pytest.importorskip("paper_2512_16512_amd")

from test_operators import BF16, U, as_type, dev, dev8, host, normal, scaled, uneven_groups, within  # noqa: E402

F32, B16 = torch.float32, torch.bfloat16
KINDS = ("fp8", "bf16", "bf16 turned", "wgrad")     # as the library numbers them

# kind, type of the result, groups (0: a product without), rows, N, K
SIZES = [
    ("fp8", F32, 0, 654, 2704, 400), ("fp8", F32, 40, 126, 1240, 400), ("fp8", F32, 16, 2600, 1608, 528),
    ("fp8", F32, 0, 6644, 136, 432), ("fp8", F32, 40, 182, 1600, 400), ("fp8", F32, 0, 10, 112, 400),
    ("fp8", F32, 0, 53, 4088, 416), ("fp8", F32, 0, 4140, 96, 416), ("fp8", F32, 3, 10, 96, 400),
    ("fp8", F32, 0, 100, 3512, 400), ("fp8", F32, 70, 220, 104, 416), ("fp8", F32, 0, 4098, 104, 400),
    ("fp8", F32, 70, 2197, 136, 400),
    ("fp8", B16, 0, 8095, 1960, 416), ("fp8", B16, 9, 7006, 4040, 448), ("fp8", B16, 0, 3520, 1672, 400),
    ("fp8", B16, 70, 3524, 328, 1424), ("fp8", B16, 0, 528, 3600, 832), ("fp8", B16, 0, 5875, 136, 416),
    ("fp8", B16, 70, 219, 232, 400), ("fp8", B16, 0, 10, 96, 448), ("fp8", B16, 0, 70, 3368, 400),
    ("fp8", B16, 0, 5502, 144, 1168), ("fp8", B16, 3, 10, 104, 560), ("fp8", B16, 0, 131, 2464, 944),
    ("fp8", B16, 70, 237, 104, 1056), ("fp8", B16, 0, 101, 3184, 400), ("fp8", B16, 3, 11, 104, 416),
    ("bf16", F32, 9, 6907, 1672, 272), ("bf16", F32, 4, 3000, 4096, 256), ("bf16", F32, 70, 238, 3312, 416),
    ("bf16", F32, 40, 124, 1344, 608), ("bf16", F32, 70, 6306, 136, 224), ("bf16", F32, 70, 261, 200, 192),
    ("bf16", F32, 3, 11, 104, 192),
    ("bf16 turned", F32, 9, 2902, 3888, 288), ("bf16 turned", F32, 70, 2689, 2440, 224),
    ("bf16 turned", F32, 17, 52, 2584, 736), ("bf16 turned", F32, 70, 6771, 136, 192),
    ("bf16 turned", F32, 70, 231, 200, 192), ("bf16 turned", F32, 3, 13, 104, 192),
    ("wgrad", F32, 40, 132, 1312, 136), ("wgrad", F32, 3, 3001, 1304, 1296), ("wgrad", F32, 40, 5603, 136, 1336),
    ("wgrad", F32, 5, 900, 96, 104),
]
# (the choice does not look at the type of a bf16 product's result)
SIZES += [(kind, B16, *size) for kind, out, *size in SIZES if kind != "fp8"]


@pytest.fixture(scope="module")
def place():
    f = ctypes.CDLL(x.LIB_PATH).xtc_test_product_kernel
    f.argtypes = [ctypes.c_int32] * 2 + [ctypes.c_int64] * 4 + [ctypes.c_int32, ctypes.POINTER(ctypes.c_int32)]

    def at(kind, out, G, T, N, K):
        n = ctypes.c_int32()
        p = f(KINDS.index(kind), int(G > 0), max(G, 1), T, N, K, int(out == B16), ctypes.byref(n))
        return p, n.value

    return at


@pytest.mark.parametrize("out", [F32, B16])
@pytest.mark.parametrize("kind", KINDS)
def test_the_sizes_reach_every_kernel(place, kind, out):
    dense, grouped, kernels = set(), set(), 0
    for k, o, G, *size in SIZES:
        if (k, o) == (kind, out):
            p, kernels = place(k, o, G, *size)
            (grouped if G else dense).add(p)
    assert dense | grouped == set(range(kernels))
    if kind == "fp8":
        # with groups all but those for products without, whose place no size with groups takes
        only = {2, 3} if out == F32 else {2, 4, 5}
        assert grouped == set(range(kernels)) - only
        assert not only & {place(kind, out, G, T, N, K)[0] for G in (1, 6, 50) for T in (1, 9, 130, 1000, 8000)
                           for N in (112, 1000, 4096) for K in (128, 1040, 4096)}


def test_rows_of_no_whole_16_bytes_take_the_kernel_for_any_address(place):
    assert place("fp8", F32, 0, 5, 8, 15)[0] == place("bf16", F32, 2, 5, 9, 8)[0] == -1


def bound(out, ref, mag, terms, eight=None):
    b = 2 * U * (terms + 8) * mag + U * ref.abs()
    if out == B16:
        b += BF16 * ref.abs()
        if eight is not None:       # (no product of a group of eight exceeds that of its operands' largest)
            b += 2.0 ** -10 * eight
    return b


def most_of_eight(v):
    return v.abs().reshape(*v.shape[:-1], v.shape[-1] // 8, 8).amax(-1)


def groups_of(G, T):
    sizes, ends = uneven_groups(T, G) if G else ([T], None)
    at = [0] + np.cumsum(sizes).tolist()
    return [(g, at[g], at[g + 1]) for g in range(len(sizes))], ends, at[-1]


@pytest.mark.gpu
@pytest.mark.parametrize("kind,out,G,T,N,K", SIZES)
def test_kernel(kind, out, G, T, N, K):
    if not torch.cuda.is_available():
        pytest.skip("no GPU visible")
    rows, ends, last = groups_of(G, T)
    what = "%s %s %s" % (kind, out, (G, T, N, K))
    say(what)
    if kind == "wgrad":
        a, dy = as_type(normal(1, T, K), "bf16"), as_type(normal(2, T, N), "bf16")
        got = host(x.matmul_grouped_wgrad(dev(a), dev(dy), ends.cuda(), dtype=out))
        for g, i, j in rows:
            p, q = a[i:j].double().t(), dy[i:j].double()
            ref = p @ q
            within(got[g], ref, bound(out, ref, p.abs() @ q.abs(), j - i), what)
        return
    if kind == "fp8":
        qa, sa, a = scaled(3, 1, T, K)
        qb, sb, b = scaled(4, 128, *((G,) if G else ()), N, K)
        if G:
            got = x.matmul_grouped_fp8(dev8(qa), dev(sa), dev8(qb), dev(sb), ends.cuda(), dtype=out)
        else:
            got, b = x.matmul_fp8(dev8(qa), dev(sa), dev8(qb), dev(sb), dtype=out), b[None]
    else:
        a, b = as_type(normal(5, T, K), "bf16"), as_type(normal(6, G, N, K), "bf16")
        stored = b if kind == "bf16 turned" else b.transpose(1, 2).contiguous()
        got = x.matmul_grouped(dev(a), dev(stored), ends.cuda(), transpose_b=kind == "bf16 turned", dtype=out)
        a, b = a.double(), b.double()
    assert got.dtype == out and got.shape == (T, N)
    got = host(got)
    for g, i, j in rows:
        ref = a[i:j] @ b[g].t()
        eight = most_of_eight(a[i:j]) @ most_of_eight(b[g]).t() if kind == "fp8" and out == B16 else None
        within(got[i:j], ref, bound(out, ref, a[i:j].abs() @ b[g].abs().t(), K, eight), what)
    assert bool((got[last:] == 0).all())


@pytest.mark.gpu
@pytest.mark.parametrize("out", [F32, B16])
def test_rows_at_any_address_of_several_tiles(out):
    """K of no multiple of 16 bytes, rows at odd elements: more than one tile of rows and of columns."""
    if not torch.cuda.is_available():
        pytest.skip("no GPU visible")
    M, N, K = 701, 903, 999
    qa, sa, a = scaled(7, 1, M, K)
    qb, sb, b = scaled(8, 128, N, K)
    pad = torch.nn.functional.pad
    say("matmul_fp8", M, N, K, out)
    got = host(x.matmul_fp8(dev8(qa, True), dev(sa, True), dev8(qb, True), dev(sb, True), dtype=out))
    ref = a @ b.t()
    eight = most_of_eight(pad(a, (0, 1))) @ most_of_eight(pad(b, (0, 1))).t()
    within(got, ref, bound(out, ref, a.abs() @ b.abs().t(), K, eight), "any address")
    rows, ends, last = groups_of(5, 2001)
    N, K = 261, 301
    a, b = as_type(normal(9, 2001, K), "bf16"), as_type(normal(10, 5, N, K), "bf16")
    dy = as_type(normal(11, 2001, N), "bf16")
    for turned in (False, True):
        say("matmul_grouped", 2001, N, K, out, turned)
        stored = b if turned else b.transpose(1, 2).contiguous()
        got = host(x.matmul_grouped(dev(a, True), dev(stored, True), ends.cuda(), transpose_b=turned, dtype=out))
        for g, i, j in rows:
            p, q = a[i:j].double(), b[g].double().t()
            ref = p @ q
            within(got[i:j], ref, bound(out, ref, p.abs() @ q.abs(), K), "any address, groups")
        assert bool((got[last:] == 0).all())
    say("matmul_grouped_wgrad", 2001, N, K, out)
    got = host(x.matmul_grouped_wgrad(dev(a, True), dev(dy, True), ends.cuda(), dtype=out))
    for g, i, j in rows:
        p, q = a[i:j].double().t(), dy[i:j].double()
        ref = p @ q
        within(got[g], ref, bound(out, ref, p.abs() @ q.abs(), j - i), "any address, weights' gradient")

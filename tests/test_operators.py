"""The norm, 8-bit and grouped operators against their definitions in 64 bits.

Tolerances.  u = 2^-24 is half a unit in the last place of fp32.  A sum of n
fp32 terms in any order is within n u of the sum of their magnitudes; the matrix
cores may truncate where they add, so products count 2u a term.  Rounding to
bf16 is within 2^-8 of the value (eight significant bits), to e4m3 within 2^-4
of it, and within half the step of its subnormals, 2^-10, near zero.  Products in
8 bits with a bf16 result may run on the 8-bit matrix instructions: of the eight
products of eight consecutive k those cut off what is below 2^-13 of the
largest's power of two, so eight times that, 2^-10 of the group's largest
magnitude, is added for each group; with an fp32 result nothing is."""
import numpy as np
import pytest

from _helpers import say

torch = pytest.importorskip("torch")
x = pytest.importorskip("paper_2512_16512_amd")

U = 2.0 ** -24
BF16 = 2.0 ** -8


@pytest.fixture(scope="module", autouse=True)
def _gpu(request):
    if not torch.cuda.is_available():
        pytest.skip("no GPU visible")


pytestmark = pytest.mark.gpu


def rng(seed):
    return torch.Generator().manual_seed(seed)


def normal(seed, *shape):
    return torch.randn(*shape, generator=rng(seed), dtype=torch.float64)


def as_type(t, dtype):
    return t.to(torch.float32 if dtype == "f32" else torch.bfloat16)


def dev(t, odd=False):
    """On the GPU; ``odd``: as the inside of a wider matrix, its rows at odd elements."""
    if not odd:
        return t.cuda()
    wide = torch.full((*t.shape[:-1], t.shape[-1] + 3), 7.0).to(t.dtype).cuda()
    wide[..., 1:1 + t.shape[-1]] = t.cuda()
    return wide[..., 1:1 + t.shape[-1]]


def host(t):
    torch.cuda.synchronize()
    return t.cpu().double()


def within(got, ref, bound, what):
    got, ref, bound = (np.asarray(v, dtype=np.float64) for v in (got, ref, bound))
    assert got.shape == ref.shape, (what, got.shape, ref.shape)
    if got.size == 0:
        return
    assert np.array_equal(np.isnan(got), np.isnan(ref)), "%s: NaN where there should be none, or none" % what
    over = np.abs(got - ref) - np.broadcast_to(bound, ref.shape)
    worst = np.nanmax(over) if not np.all(np.isnan(over)) else -1.0
    assert worst <= 0, "%s: %g over its bound" % (what, worst)


def blocks(y, rows):
    """Scale of each value's block, and the block scales, by the definition."""
    M, K = y.shape
    kb, mb = -(-K // 128), -(-M // rows)
    s = torch.zeros(mb, kb, dtype=torch.float64)
    each = torch.zeros(M, K, dtype=torch.float64)
    for i in range(mb):
        for j in range(kb):
            cut = y[i * rows:(i + 1) * rows, j * 128:(j + 1) * 128]
            fine = cut[torch.isfinite(cut)].abs()
            s[i, j] = max((fine.max().item() if fine.numel() else 0.0) / 448, 2.0 ** -126)
            each[i * rows:(i + 1) * rows, j * 128:(j + 1) * 128] = s[i, j]
    return each, s


def check_e4m3(q, scale, y, rows, rel, what):
    """``q`` and ``scale`` stand for ``y``, which is itself within ``rel`` of the kernel's."""
    each, s = blocks(y, rows)
    within(host(scale), s, (rel + 4 * U) * s, what + " scale")
    want = torch.where(torch.isfinite(y), y / each, float("nan"))
    got = host(q.float())
    within(got, want, want.abs() * (2.0 ** -4 + 2 * rel + 8 * U) + 2.0 ** -10, what)


SIZES = [(1, 1), (3, 7), (2, 127), (5, 128), (4, 129), (1, 4096), (33, 512), (7, 1021), (3, 2050), (2, 8192), (1, 8200),
         (2, 20001), (1, 40000)]


# ------------------------------------------------------------------ norm


def norm_case(T, D, dtype, residual, seed):
    xs = as_type(normal(seed, T, D) * torch.exp(normal(seed + 1, D)), dtype)
    w = as_type(1 + 0.2 * normal(seed + 2, D), dtype)
    r = as_type(3 * normal(seed + 3, T, D), dtype) if residual else None
    return xs, w, r


def norm_reference(xs, w, r, eps):
    h = xs.double() + (r.double() if r is not None else 0)
    rstd = 1 / torch.sqrt(h.square().mean(1) + eps)
    return h, rstd, w.double() * h * rstd[:, None]


@pytest.mark.parametrize("quantize", [False, True])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T,D", SIZES)
def test_rmsnorm(T, D, dtype, quantize):
    for residual in (False, True):
        xs, w, r = norm_case(T, D, dtype, residual, 10 * D + T)
        h, rstd, y = norm_reference(xs, w, r, 1e-5)
        rel = (D + 16) * U
        tail = BF16 if dtype == "bf16" else U
        for odd in (False, True):
            what = "rmsnorm %s" % ((T, D, dtype, quantize, residual, odd),)
            say(what)
            n = x.rmsnorm(dev(xs, odd), dev(w), None if r is None else dev(r, odd), eps=1e-5, quantize=quantize)
            within(host(n.rstd), rstd, rel * rstd, what + " rstd")
            if residual:
                assert n.residual.dtype == xs.dtype
                within(host(n.residual), h, tail * h.abs() + U * (xs.double().abs() + r.double().abs()), what + " sum")
            if quantize:
                assert n.out.dtype == torch.float8_e4m3fn and n.scale.shape == (T, -(-D // 128))
                check_e4m3(n.out, n.scale, y, 1, rel, what)
            else:
                assert n.scale is None and n.out.dtype == xs.dtype
                within(host(n.out), y, (tail + 2 * rel) * y.abs(), what)


def test_rmsnorm_weight_in_32_bits_and_rows_of_zeros():
    xs = as_type(normal(1, 6, 300), "bf16")
    xs[2] = 0
    w = normal(2, 300).float()
    _, rstd, y = norm_reference(xs, w, None, 1e-6)
    n = x.rmsnorm(dev(xs), dev(w))
    within(host(n.out), y, (BF16 + 700 * U) * y.abs(), "fp32 weight")
    within(host(n.rstd), rstd, 316 * U * rstd, "rstd")
    q = x.rmsnorm(dev(xs), dev(w), quantize=True)
    assert bool((q.out[2].float() == 0).all()) and bool((q.scale[2] == 2.0 ** -126).all())


def test_rmsnorm_not_finite_values_stay_in_their_row():
    xs = normal(3, 5, 260).float()
    xs[1, 7], xs[3, 130] = float("nan"), float("inf")
    w = torch.ones(260)
    n = x.rmsnorm(dev(xs), dev(w), quantize=True)
    plain = x.rmsnorm(dev(xs), dev(w))
    for t in (0, 2, 4):
        assert bool(torch.isfinite(n.out[t].float()).all()) and bool(torch.isfinite(plain.out[t]).all())
    assert bool(torch.isnan(plain.out[1]).all()) and bool(torch.isnan(n.out[1].float()).all())
    # an infinite sum of squares: rstd is 0, the infinite value 0 * inf
    assert bool(torch.isnan(plain.out[3, 130])) and bool((plain.out[3, :130] == 0).all())
    assert bool(torch.isnan(n.out[3, 130].float())) and bool((n.out[3, :130].float() == 0).all())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T,D", [(0, 64), (1, 1), (1, 4096), (3, 129), (600, 40), (1030, 257), (37, 2050), (513, 1024),
                                 (2, 20001)])
def test_rmsnorm_backward(T, D, dtype):
    for residual in (False, True):
        xs, w, _ = norm_case(T, D, dtype, False, 7 * D + T)
        dy = as_type(normal(D, T, D), dtype)
        dr = as_type(normal(D + 1, T, D), dtype) if residual else None
        rstd = (1 / torch.sqrt(xs.double().square().mean(1) + 1e-6)).float()
        xh = xs.double() * rstd.double()[:, None]
        g = dy.double() * w.double()
        mean = (g * xh).mean(1, keepdim=True)
        dx = rstd.double()[:, None] * (g - xh * mean) + (dr.double() if residual else 0)
        dw = (dy.double() * xh).sum(0)
        size = rstd.double()[:, None] * (g.abs() + xh.abs() * (g * xh).abs().mean(1, keepdim=True) * (D + 8))
        tail = BF16 if dtype == "bf16" else U
        for odd in (False, True):
            what = "rmsnorm_backward %s" % ((T, D, dtype, residual, odd),)
            say(what)
            gx, gw = x.rmsnorm_backward(dev(dy, odd), dev(xs, odd), dev(w), dev(rstd),
                                        None if dr is None else dev(dr, odd))
            assert gx.dtype == xs.dtype and gw.dtype == torch.float32
            within(host(gx), dx, tail * dx.abs() + 8 * U * (size + (dr.double().abs() if residual else 0)), what + " dx")
            within(host(gw), dw, (T + 8) * U * (dy.double() * xh).abs().sum(0), what + " dweight")


def test_rmsnorm_backward_against_differences():
    """Central differences of the 64-bit forward along random directions: their own error is about step^2."""
    T, D, eps, step = 9, 333, 1e-6, 1e-5
    xs, w = normal(1, T, D).float(), (1 + 0.3 * normal(2, D)).float()
    dy = normal(3, T, D).float()
    n = x.rmsnorm(dev(xs), dev(w), eps=eps)
    dx, dw = (host(t) for t in x.rmsnorm_backward(dev(dy), dev(xs), dev(w), n.rstd))

    def loss(a, b):
        return (norm_reference(a, b, None, eps)[2] * dy.double()).sum().item()

    for seed in range(4):
        v, u = normal(20 + seed, T, D), normal(30 + seed, D)
        a, b = xs.double(), w.double()
        num = (loss(a + step * v, b) - loss(a - step * v, b)) / (2 * step)
        assert abs(num - (dx * v).sum().item()) <= 1e-4 * (dx * v).norm().item() * 10
        num = (loss(a, b + step * u) - loss(a, b - step * u)) / (2 * step)
        assert abs(num - (dw * u).sum().item()) <= 1e-4 * (dw * u).norm().item() * 10


def test_rmsnorm_backward_gives_the_same_bits_again():
    xs, w, _ = norm_case(777, 1030, "bf16", False, 5)
    dy = dev(as_type(normal(6, 777, 1030), "bf16"))
    n = x.rmsnorm(dev(xs), dev(w))
    first = x.rmsnorm_backward(dy, dev(xs), dev(w), n.rstd)
    for _ in range(3):
        again = x.rmsnorm_backward(dy, dev(xs), dev(w), n.rstd)
        assert torch.equal(first[0], again[0]) and torch.equal(first[1], again[1])


# ------------------------------------------------------------ quantize_fp8


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows", [1, 128])
@pytest.mark.parametrize("M,K", [(0, 5), (1, 1), (3, 128), (130, 129), (128, 256), (257, 1000), (5, 4096)])
def test_quantize(M, K, rows, dtype):
    v = as_type(normal(M * 1000 + K, M, K) * torch.exp(2 * normal(4, K)), dtype)
    for odd in (False, True):
        say("quantize_fp8", M, K, rows, dtype, odd)
        q, s = x.quantize_fp8(dev(v, odd), block_rows=rows)
        assert q.shape == (M, K) and s.shape == (-(-M // rows), -(-K // 128))
        check_e4m3(q, s, v.double(), rows, 0.0, "quantize")


@pytest.mark.parametrize("rows", [1, 128])
def test_quantize_extremes(rows):
    v = torch.zeros(4, 640)
    v[0, 0], v[0, 1], v[0, 2] = 3.0, float("nan"), float("-inf")     # keep the others' values
    v[1, 128:256] = 1e-40                                              # below the least scale
    v[2, 256:384] = 3e38
    v[3, 384] = 448.0
    v[3, 385:400] = torch.linspace(-448, 448, 15)
    q, s = x.quantize_fp8(dev(v), block_rows=rows)
    check_e4m3(q, s, v.double(), rows, 0.0, "extremes")
    assert bool((s[:, 4] == 2.0 ** -126).all())


def test_quantize_every_e4m3_value_comes_back():
    bits = torch.arange(256, dtype=torch.uint8)
    v = bits.view(torch.float8_e4m3fn).float()
    v = torch.where(torch.isnan(v), torch.tensor(448.0), v).reshape(2, 128)
    q, s = x.quantize_fp8(dev(v))
    assert bool((s == 1).all()) and torch.equal(q.float().cpu(), v)


# ---------------------------------------------------------- 8-bit products


def scaled(seed, rows, *shape):
    """An e4m3 operand with its scales, and the values it stands for in 64 bits."""
    *lead, M, K = shape
    mb, kb = -(-M // rows), -(-K // 128)
    q = (normal(seed, *shape) * 60).clamp(-448, 448).float().to(torch.float8_e4m3fn)
    s = torch.exp(normal(seed + 1, *lead, mb, kb)).float()
    each = s.double().repeat_interleave(rows, -2)[..., :M, :].repeat_interleave(128, -1)[..., :K]
    return q, s, q.double() * each


def cut_off(a, b):
    """The 8-bit instructions' bound for a [M, K] and b [K, N]: 2^-10 of the largest product of each eight k."""
    K = a.shape[-1]
    a, b = a.abs(), b.abs()
    pad = -K % 8
    a = torch.nn.functional.pad(a, (0, pad)).reshape(a.shape[0], -1, 8)
    b = torch.nn.functional.pad(b.t(), (0, pad)).reshape(b.shape[1], -1, 8)
    total = torch.zeros(a.shape[0], b.shape[0], dtype=torch.float64)
    for g in range(a.shape[1]):
        total += (a[:, None, g] * b[None, :, g]).amax(-1)
    return 2.0 ** -10 * total


def product_bound(a, b, K, out):
    ref = a @ b
    if out == torch.bfloat16:
        return ref, 2 * U * (K + 8) * (a.abs() @ b.abs()) + BF16 * ref.abs() + cut_off(a, b)
    return ref, 2 * U * (K + 8) * (a.abs() @ b.abs()) + (BF16 if out == torch.bfloat16 else U) * ref.abs()


FP8_SIZES = [(1, 1, 1), (1, 128, 128), (2, 3, 127), (7, 130, 129), (16, 256, 512), (17, 129, 1000), (64, 64, 64),
             (100, 300, 640), (1, 2048, 1024), (5, 1000, 2047), (33, 512, 2048), (130, 260, 1030), (257, 513, 384),
             (300, 1024, 256)]


@pytest.mark.parametrize("M,N,K", FP8_SIZES)
def test_matmul_fp8(M, N, K):
    qa, sa, a = scaled(M + K, 1, M, K)
    qb, sb, b = scaled(N + K + 7, 128, N, K)
    for out in (torch.float32, torch.bfloat16):
        ref, bound = product_bound(a, b.t(), K, out)
        for odd in (False, True):
            say("matmul_fp8", M, N, K, out, odd)
            got = x.matmul_fp8(dev8(qa, odd), dev(sa, odd), dev8(qb, odd), dev(sb, odd), dtype=out)
            assert got.dtype == out
            within(host(got), ref, bound, "matmul_fp8")
    got = x.matmul_fp8(dev8(qa), dev(sa), dev8(qb), dev(sb), relu=True)
    ref, bound = product_bound(a, b.t(), K, torch.float32)
    within(host(got), ref.clamp_min(0), bound, "relu")


def dev8(q, odd=False):
    """Like dev() for 8-bit values (their bytes moved)."""
    return dev(q.view(torch.uint8), odd).view(torch.float8_e4m3fn)


def test_matmul_fp8_writes_its_own_columns_only():
    qa, sa, a = scaled(1, 1, 37, 200)
    qb, sb, b = scaled(2, 128, 150, 200)
    wide = torch.full((37, 163), 5.0, device="cuda")
    got = x.matmul_fp8(dev8(qa), dev(sa), dev8(qb), dev(sb), out=wide[:, 3:153])
    ref, bound = product_bound(a, b.t(), 200, torch.float32)
    within(host(got), ref, bound, "out")
    assert bool((wide[:, :3] == 5).all()) and bool((wide[:, 153:] == 5).all())


@pytest.mark.parametrize("M,N,K", [(4, 0, 8), (0, 4, 8), (3, 5, 0)])
def test_matmul_fp8_empty(M, N, K):
    qa, sa, _ = scaled(1, 1, M, K)
    qb, sb, _ = scaled(2, 128, N, K)
    got = x.matmul_fp8(dev8(qa), dev(sa), dev8(qb), dev(sb))
    assert got.shape == (M, N) and bool((got == 0).all())


@pytest.mark.parametrize("M", [3, 200])
def test_matmul_fp8_nan_stays_in_its_row_and_column(M):
    """A NaN behind the end of k, or in another row, does not reach a result."""
    K, N = 136, 140
    qa, sa, a = scaled(1, 1, M, K + 16)
    qb, sb, b = scaled(2, 128, N, K + 16)
    nan = torch.tensor([0x7F], dtype=torch.uint8)
    qa.view(torch.uint8)[:, K:] = nan
    qb.view(torch.uint8)[:, K:] = nan
    qa.view(torch.uint8)[1, 5] = nan
    qb.view(torch.uint8)[77, 130] = nan
    got = host(x.matmul_fp8(dev8(qa)[:, :K], dev(sa), dev8(qb)[:, :K], dev(sb)))
    a, b = (q[:, :K].double() * s.double().repeat_interleave(r, 0)[:q.shape[0]].repeat_interleave(128, 1)[:, :K]
            for q, s, r in ((qa, sa, 1), (qb, sb, 128)))
    ref, bound = product_bound(a, b.t(), K, torch.float32)
    assert bool(torch.isnan(ref[1]).all()) and bool(torch.isnan(ref[:, 77]).all()) and int(torch.isnan(ref).sum()) == M + N - 1
    within(got, ref, torch.where(torch.isnan(bound), torch.zeros(()).double(), bound), "nan")
    relu = host(x.matmul_fp8(dev8(qa)[:, :K], dev(sa), dev8(qb)[:, :K], dev(sb), relu=True))
    assert torch.equal(torch.isnan(relu), torch.isnan(ref))


# ----------------------------------------------------------------- groups


GROUPS = {
    "one": [5],
    "some empty": [0, 3, 0, 0, 20, 1, 0],
    "tail without a group": [4, 9, -6],          # the last is the rows that belong to none
    "none at all": [0, 0, 0, -10],
    "ragged": [130, 1, 64, 257, 16, 0, 33],
    "many": [(7 * i) % 5 for i in range(150)],
}


def group_rows(name):
    sizes = [n for n in GROUPS[name] if n >= 0]
    T = sum(abs(n) for n in GROUPS[name])
    return T, sizes, torch.tensor(np.cumsum(sizes), dtype=torch.int32)


def grouped_reference(a, b, sizes):
    ref = torch.zeros(a.shape[0], b.shape[2], dtype=torch.float64)
    i = 0
    for g, n in enumerate(sizes):
        ref[i:i + n] = a[i:i + n] @ b[g]
        i += n
    return ref


@pytest.mark.parametrize("transpose_b", [False, True])
@pytest.mark.parametrize("N,K", [(1, 1), (64, 64), (129, 70), (256, 128), (40, 520), (264, 136)])
@pytest.mark.parametrize("name", list(GROUPS))
def test_matmul_grouped(name, N, K, transpose_b):
    T, sizes, ends = group_rows(name)
    a, b = as_type(normal(K, T, K), "bf16"), as_type(normal(N, len(sizes), K, N), "bf16")
    ref = grouped_reference(a.double(), b.double(), sizes)
    mag = grouped_reference(a.double().abs(), b.double().abs(), sizes)
    stored = b.transpose(1, 2).contiguous() if transpose_b else b
    for out in (torch.float32, torch.bfloat16):
        for odd in (False, True):
            say("matmul_grouped", name, N, K, transpose_b, out, odd)
            got = x.matmul_grouped(dev(a, odd), dev(stored, odd), ends.cuda(), transpose_b=transpose_b, dtype=out)
            assert got.dtype == out
            within(host(got), ref, 2 * U * (K + 8) * mag + (BF16 if out == torch.bfloat16 else U) * ref.abs(), "grouped")
    got = x.matmul_grouped(dev(a), dev(stored), ends.cuda(), transpose_b=transpose_b, relu=True)
    within(host(got), ref.clamp_min(0), 2 * U * (K + 8) * mag + U * ref.abs(), "relu")


@pytest.mark.parametrize("N,K", [(1, 1), (64, 64), (129, 70), (264, 136)])
@pytest.mark.parametrize("name", list(GROUPS))
def test_matmul_grouped_wgrad(name, N, K):
    T, sizes, ends = group_rows(name)
    a, dy = as_type(normal(K, T, K), "bf16"), as_type(normal(N, T, N), "bf16")
    ref, mag = (torch.zeros(len(sizes), K, N, dtype=torch.float64) for _ in range(2))
    i = 0
    for g, n in enumerate(sizes):
        ref[g] = a[i:i + n].double().t() @ dy[i:i + n].double()
        mag[g] = a[i:i + n].double().abs().t() @ dy[i:i + n].double().abs()
        i += n
    for out in (torch.float32, torch.bfloat16):
        for odd in (False, True):
            say("matmul_grouped_wgrad", name, N, K, out, odd)
            got = x.matmul_grouped_wgrad(dev(a, odd), dev(dy, odd), ends.cuda(), dtype=out)
            tail = BF16 if out == torch.bfloat16 else U
            within(host(got), ref, 2 * U * (max(sizes) + 8) * mag + tail * ref.abs(), "wgrad")


def test_grouped_gradients_against_differences():
    """The product is linear in each operand, so the loss's differences are exact but for the rounding of the gradients' fp32 sums."""
    T, sizes, ends = group_rows("ragged")
    N, K = 72, 104
    a, b = as_type(normal(1, T, K), "bf16"), as_type(normal(2, len(sizes), K, N), "bf16")
    dy = as_type(normal(3, T, N), "bf16")
    da = host(x.matmul_grouped(dev(dy), dev(b), ends.cuda(), transpose_b=True))
    db = host(x.matmul_grouped_wgrad(dev(a), dev(dy), ends.cuda()))

    def loss(p, q):
        return (grouped_reference(p, q, sizes) * dy.double()).sum().item()

    for seed in range(3):
        v, u = normal(40 + seed, T, K), normal(50 + seed, len(sizes), K, N)
        p, q = a.double(), b.double()
        num = (loss(p + v, q) - loss(p - v, q)) / 2
        assert abs(num - (da * v).sum().item()) <= 1e-5 * (da.abs() * v.abs()).sum().item()
        num = (loss(p, q + u) - loss(p, q - u)) / 2
        assert abs(num - (db * u).sum().item()) <= 1e-5 * (db.abs() * u.abs()).sum().item()


@pytest.mark.parametrize("N,K", [(1, 1), (64, 128), (130, 200), (256, 384), (512, 1024)])
@pytest.mark.parametrize("name", list(GROUPS))
def test_matmul_grouped_fp8(name, N, K):
    T, sizes, ends = group_rows(name)
    qa, sa, a = scaled(K, 1, T, K)
    qb, sb, b = scaled(N + 3, 128, len(sizes), N, K)
    ref = grouped_reference(a, b.transpose(1, 2), sizes)
    mag = grouped_reference(a.abs(), b.abs().transpose(1, 2), sizes)
    cut, i = torch.zeros_like(ref), 0
    for g, n in enumerate(sizes):
        cut[i:i + n] = cut_off(a[i:i + n], b[g].t()) if n else 0
        i += n
    for out in (torch.float32, torch.bfloat16):
        for odd in (False, True):
            say("matmul_grouped_fp8", name, N, K, out, odd)
            got = x.matmul_grouped_fp8(dev8(qa, odd), dev(sa, odd), dev8(qb, odd), dev(sb, odd), ends.cuda(), dtype=out)
            bf16 = out == torch.bfloat16
            within(host(got), ref, 2 * U * (K + 8) * mag + (BF16 if bf16 else U) * ref.abs() + (cut if bf16 else 0), "fp8")
    got = x.matmul_grouped_fp8(dev8(qa), dev(sa), dev8(qb), dev(sb), ends.cuda(), relu=True)
    within(host(got), ref.clamp_min(0), 2 * U * (K + 8) * mag + U * ref.abs(), "relu")


def test_grouped_ends_that_do_not_ascend_stay_in_range():
    """A value below an earlier one makes an empty group, one past T counts as T."""
    T, N, K = 70, 48, 64
    a, b = as_type(normal(1, T, K), "bf16"), as_type(normal(2, 5, K, N), "bf16")
    dy = as_type(normal(3, T, N), "bf16")
    sizes = [0, 30, 0, 40, 0]
    ref = grouped_reference(a.double(), b.double(), sizes)
    ends = torch.tensor([-5, 30, 11, 1000, 60], dtype=torch.int32)
    got = host(x.matmul_grouped(dev(a), dev(b), ends.cuda()))
    within(got, ref, 2 * U * (K + 8) * grouped_reference(a.double().abs(), b.double().abs(), sizes), "ends")
    dw = host(x.matmul_grouped_wgrad(dev(a), dev(dy), ends.cuda()))
    want = torch.zeros(5, K, N, dtype=torch.float64)
    want[1], want[3] = a[:30].double().t() @ dy[:30].double(), a[30:].double().t() @ dy[30:].double()
    within(dw, want, 2 * U * 80 * (a.double().abs().t() @ dy.double().abs()), "wgrad")


def test_grouped_not_finite_rows_stay_in_their_group():
    T, sizes, ends = group_rows("ragged")
    N, K = 136, 72
    a, b = as_type(normal(1, T, K), "bf16"), as_type(normal(2, len(sizes), K, N), "bf16")
    dy = as_type(normal(3, T, N), "bf16")
    a[131:195] = float("nan")                  # the third group's rows
    b[3] = float("inf")                        # and the fourth's matrix
    got = host(x.matmul_grouped(dev(a), dev(b), ends.cuda()))
    bad = torch.zeros(T, dtype=torch.bool)
    bad[131:195 + 257] = True
    assert bool(torch.isfinite(got[~bad]).all()) and not bool(torch.isfinite(got[bad]).any())
    dw = host(x.matmul_grouped_wgrad(dev(a), dev(dy), ends.cuda()))
    assert bool(torch.isnan(dw[2]).all()) and bool(torch.isfinite(dw[[0, 1, 3, 4, 5, 6]]).all())
    assert bool((dw[5] == 0).all())


# Sizes at which the products take their large tiles and a workgroup computes
# more than one of them.


@pytest.mark.parametrize("out", [torch.float32, torch.bfloat16])
def test_matmul_fp8_large_tiles(out):
    M, N, K = 4099, 4000, 400
    qa, sa, a = scaled(5, 1, M, K)
    qb, sb, b = scaled(6, 128, N, K)
    say("matmul_fp8", M, N, K, out)
    got = host(x.matmul_fp8(dev8(qa), dev(sa), dev8(qb), dev(sb), dtype=out))
    ref = a @ b.t()
    bound = 2 * U * (K + 8) * (a.abs() @ b.abs().t())
    if out == torch.bfloat16:
        # no product of a group of eight exceeds the product of its operands' largest
        eight = [v.abs().reshape(v.shape[0], K // 8, 8).amax(2) for v in (a, b)]
        bound += BF16 * ref.abs() + 2.0 ** -10 * (eight[0] @ eight[1].t())
    within(got, ref, bound + U * ref.abs(), "large tiles")


LARGE_SIZES = [1500, 0, 2100, 7, 3000, 256, 900, 1, 800, -436]


def large_groups():
    T = sum(abs(n) for n in LARGE_SIZES)
    sizes = [n for n in LARGE_SIZES if n >= 0]
    return T, sizes, torch.tensor(np.cumsum(sizes), dtype=torch.int32)


@pytest.mark.parametrize("transpose_b", [False, True])
def test_matmul_grouped_large_tiles(transpose_b):
    T, sizes, ends = large_groups()
    N, K = 2088, 200
    a, b = as_type(normal(1, T, K), "bf16"), as_type(normal(2, len(sizes), K, N), "bf16")
    stored = b.transpose(1, 2).contiguous() if transpose_b else b
    ref = grouped_reference(a.double(), b.double(), sizes)
    mag = grouped_reference(a.double().abs(), b.double().abs(), sizes)
    for out in (torch.float32, torch.bfloat16):
        say("matmul_grouped", T, N, K, transpose_b, out)
        got = host(x.matmul_grouped(dev(a), dev(stored), ends.cuda(), transpose_b=transpose_b, dtype=out))
        within(got, ref, 2 * U * (K + 8) * mag + (BF16 if out == torch.bfloat16 else U) * ref.abs(), "large tiles")


def test_matmul_grouped_fp8_large_tiles():
    T, sizes, ends = large_groups()
    N, K = 2100, 272
    qa, sa, a = scaled(8, 1, T, K)
    qb, sb, b = scaled(9, 128, len(sizes), N, K)
    ref = grouped_reference(a, b.transpose(1, 2), sizes)
    mag = grouped_reference(a.abs(), b.abs().transpose(1, 2), sizes)
    eight = [v.abs().reshape(*v.shape[:-1], K // 8, 8).amax(-1) for v in (a, b)]
    cut = 2.0 ** -10 * grouped_reference(eight[0], eight[1].transpose(1, 2), sizes)
    say("matmul_grouped_fp8", T, N, K)
    got = host(x.matmul_grouped_fp8(dev8(qa), dev(sa), dev8(qb), dev(sb), ends.cuda(), dtype=torch.bfloat16))
    within(got, ref, 2 * U * (K + 8) * mag + BF16 * ref.abs() + cut, "large tiles")


def test_matmul_grouped_wgrad_large_tiles():
    T, sizes, ends = large_groups()
    N, K = 1304, 1296
    a, dy = as_type(normal(1, T, K), "bf16"), as_type(normal(2, T, N), "bf16")
    say("matmul_grouped_wgrad", T, N, K)
    got = host(x.matmul_grouped_wgrad(dev(a), dev(dy), ends.cuda()))
    i = 0
    for g, n in enumerate(sizes):
        p, q = a[i:i + n].double(), dy[i:i + n].double()
        ref = p.t() @ q
        within(got[g], ref, 2 * U * (n + 8) * (p.abs().t() @ q.abs()) + U * ref.abs(), "wgrad of group %d" % g)
        i += n


# Sizes at which each of the other kernels is taken.


@pytest.mark.parametrize("quantize", [False, True])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T,D", [(5, 2048), (6, 1501)])
def test_rmsnorm_of_other_widths(T, D, dtype, quantize):
    test_rmsnorm(T, D, dtype, quantize)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T,D", [(40, 2048), (9, 8192), (270, 5001)])
def test_rmsnorm_backward_of_other_widths(T, D, dtype):
    test_rmsnorm_backward(T, D, dtype)


@pytest.mark.parametrize("M,N,K,out", [(1947, 8119, 400, torch.bfloat16), (11035, 132, 880, torch.bfloat16),
                                       (4232, 102, 160, torch.float32), (8248, 105, 160, torch.float32)])
def test_matmul_fp8_other_tiles(M, N, K, out):
    qa, sa, a = scaled(15, 1, M, K)
    qb, sb, b = scaled(16, 128, N, K)
    say("matmul_fp8", M, N, K, out)
    got = host(x.matmul_fp8(dev8(qa), dev(sa), dev8(qb), dev(sb), dtype=out))
    ref = a @ b.t()
    bound = 2 * U * (K + 8) * (a.abs() @ b.abs().t()) + U * ref.abs()
    if out == torch.bfloat16:
        eight = [v.abs().reshape(v.shape[0], K // 8, 8).amax(2) for v in (a, b)]
        bound += BF16 * ref.abs() + 2.0 ** -10 * (eight[0] @ eight[1].t())
    within(got, ref, bound, "other tiles")


def uneven_groups(T, G):
    """T rows in G groups of very different sizes, some empty, some rows past the last."""
    share = normal(T, G + 1).exp().square()
    share[::5] = 0
    share[-1] = share.sum() / 50
    sizes = (share / share.sum() * T).floor().long().tolist()
    return sizes[:G], torch.tensor(np.cumsum(sizes[:G]), dtype=torch.int32)


@pytest.mark.parametrize("T,N,K,G,transpose_b", [(10588, 392, 160, 56, False), (6836, 136, 208, 48, False),
                                                 (15549, 139, 320, 40, True), (8221, 136, 192, 2, True),
                                                 (18996, 585, 288, 22, True)])
def test_matmul_grouped_other_tiles(T, N, K, G, transpose_b):
    sizes, ends = uneven_groups(T, G)
    a, b = as_type(normal(21, T, K), "bf16"), as_type(normal(22, G, K, N), "bf16")
    stored = b.transpose(1, 2).contiguous() if transpose_b else b
    ref = grouped_reference(a.double(), b.double(), sizes)
    mag = grouped_reference(a.double().abs(), b.double().abs(), sizes)
    for out in (torch.float32, torch.bfloat16):
        say("matmul_grouped", T, N, K, G, transpose_b, out)
        got = host(x.matmul_grouped(dev(a), dev(stored), ends.cuda(), transpose_b=transpose_b, dtype=out))
        within(got, ref, 2 * U * (K + 8) * mag + (BF16 if out == torch.bfloat16 else U) * ref.abs(), "other tiles")


def test_matmul_grouped_wgrad_other_tiles():
    T, N, K, G = 205, 136, 1952, 32
    sizes, ends = uneven_groups(T, G)
    a, dy = as_type(normal(23, T, K), "bf16"), as_type(normal(24, T, N), "bf16")
    say("matmul_grouped_wgrad", T, N, K, G)
    got = host(x.matmul_grouped_wgrad(dev(a), dev(dy), ends.cuda()))
    i = 0
    for g, n in enumerate(sizes):
        p, q = a[i:i + n].double(), dy[i:i + n].double()
        ref = p.t() @ q
        within(got[g], ref, 2 * U * (n + 8) * (p.abs().t() @ q.abs()) + U * ref.abs(), "wgrad of group %d" % g)
        i += n


@pytest.mark.parametrize("T,N,K,G", [(216, 136, 920, 57), (143, 3824, 2056, 1)])
def test_matmul_grouped_wgrad_tall_and_wide(T, N, K, G):
    sizes, ends = uneven_groups(T, G) if G > 1 else ([T], torch.tensor([T], dtype=torch.int32))
    a, dy = as_type(normal(25, T, K), "bf16"), as_type(normal(26, T, N), "bf16")
    say("matmul_grouped_wgrad", T, N, K, G)
    got = host(x.matmul_grouped_wgrad(dev(a), dev(dy), ends.cuda()))
    i = 0
    for g, n in enumerate(sizes):
        p, q = a[i:i + n].double(), dy[i:i + n].double()
        ref = p.t() @ q
        within(got[g], ref, 2 * U * (n + 8) * (p.abs().t() @ q.abs()) + U * ref.abs(), "wgrad of group %d" % g)
        i += n


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("M,N", [(300, 261), (1947, 2111)])
def test_tiles_write_their_own_columns_only(M, N, dtype):
    """Results of tiles in rows that begin at odd addresses, beside columns that stay."""
    K = 400
    qa, sa, a = scaled(31, 1, M, K)
    qb, sb, b = scaled(32, 128, N, K)
    wide = torch.full((M, N + 10), 5.0, device="cuda", dtype=dtype)
    say("matmul_fp8", M, N, K, dtype)
    got = x.matmul_fp8(dev8(qa), dev(sa), dev8(qb), dev(sb), dtype=dtype, out=wide[:, 3:N + 3])
    ref = a @ b.t()
    bound = 2 * U * (K + 8) * (a.abs() @ b.abs().t()) + U * ref.abs()
    if dtype == torch.bfloat16:
        eight = [v.abs().reshape(v.shape[0], K // 8, 8).amax(2) for v in (a, b)]
        bound += BF16 * ref.abs() + 2.0 ** -10 * (eight[0] @ eight[1].t())
    within(host(got), ref, bound, "out")
    assert bool((wide[:, :3] == 5).all()) and bool((wide[:, N + 3:] == 5).all())


# Rows beyond what a launch holds at once: each workgroup of the gradient takes
# several, and the last trip is a partial one.


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T,D", [(9001, 40), (7001, 600), (2501, 1100), (2301, 2100), (601, 5001), (1201, 8200)])
def test_rmsnorm_backward_of_many_rows(T, D, dtype):
    test_rmsnorm_backward(T, D, dtype)


@pytest.mark.parametrize("quantize", [False, True])
def test_rmsnorm_of_more_rows_than_one_launch(quantize):
    """A launch holds 2^21 workgroups of four rows: the rows behind it are normed by another."""
    T, D, first = (1 << 23) + 7, 3, (1 << 23) - 6
    v = torch.zeros(T, D, device="cuda")
    r = torch.zeros(T, D, device="cuda")
    xs, w, res = norm_case(T - first, D, "f32", True, 9)
    v[first:], r[first:] = xs.cuda(), res.cuda()
    say("rmsnorm", T, D, quantize)
    n = x.rmsnorm(v, dev(w), r, eps=1e-5, quantize=quantize)
    h, rstd, y = norm_reference(xs, w, res, 1e-5)
    rel = (D + 16) * U
    within(host(n.rstd[first:]), rstd, rel * rstd, "rstd")
    within(host(n.residual[first:]), h, U * h.abs() + U * (xs.double().abs() + res.double().abs()), "sum")
    if quantize:
        check_e4m3(n.out[first:], n.scale[first:], y, 1, rel, "last rows")
        assert bool((n.out[:first].view(torch.uint8) == 0).all()) and bool((n.scale[:first] == 2.0 ** -126).all())
    else:
        within(host(n.out[first:]), y, (U + 2 * rel) * y.abs(), "last rows")
        assert bool((n.out[:first] == 0).all())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows", [1, 128])
def test_quantize_divides_as_the_definition_does(rows, dtype):
    """Scales and values are the bits of fp32 divisions, amax / 448 and x / scale, the latter rounded to nearest even."""
    M, K = 384, 1280
    v = as_type(normal(77, M, K) * torch.exp(2 * normal(78, K)), dtype)
    q, s = x.quantize_fp8(dev(v), block_rows=rows)
    cut = v.float().reshape(M // rows, rows, K // 128, 128)
    scale = cut.abs().amax((1, 3)) / torch.full((), 448.0)
    assert torch.equal(s.cpu(), scale)
    want = (cut / scale[:, None, :, None]).reshape(M, K).to(torch.float8_e4m3fn)
    assert torch.equal(q.cpu().view(torch.uint8), want.view(torch.uint8))


# ------------------------------------------------------- streams, far offsets


def test_operators_run_on_the_current_stream():
    """Each call is enqueued behind what the current stream holds, and before what follows on it."""
    s = torch.cuda.Stream()
    src = normal(1, 256, 512).bfloat16().cuda()
    w = torch.ones(512, dtype=torch.bfloat16, device="cuda")
    wb = (normal(2, 128, 512) / 20).bfloat16().cuda()
    ends = torch.tensor([100, 256], dtype=torch.int32, device="cuda")
    wg = (normal(3, 2, 512, 64) / 20).bfloat16().cuda()
    torch.cuda.synchronize()

    def chain(v):
        n = x.rmsnorm(v, w, v, quantize=True)
        qb, sb = x.quantize_fp8(wb, block_rows=128)
        y = x.matmul_fp8(n.out, n.scale, qb, sb)
        z = x.matmul_grouped(n.residual, wg, ends)
        dx, dw = x.rmsnorm_backward(v, n.residual, w, n.rstd)
        return y, z, x.matmul_grouped_wgrad(v, n.residual, ends), dx, dw

    want = [t.clone() for t in chain(src)]
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        torch.cuda._sleep(20_000_000)
        v = src * 1
        got = chain(v)
        after = [t * 1 for t in got]
    s.synchronize()
    for p, q in zip(want, after):
        assert torch.equal(p, q)


def test_rows_and_matrices_past_32_bit_offsets():
    """Operands of more than 2^32 bytes: the last rows and the last matrix are the right ones."""
    K, N, G = 4096, 4096, 140
    b = torch.empty(G, K, N, dtype=torch.bfloat16, device="cuda")            # 4.7 GB
    last = (normal(1, K, N) / 64).bfloat16()
    b[-1] = last.cuda()
    T = 600_000
    a = torch.empty(T, K, dtype=torch.bfloat16, device="cuda")               # 4.9 GB
    rows = normal(2, 40, K).bfloat16()
    a[-40:] = rows.cuda()
    ends = torch.full((G,), T - 40, dtype=torch.int32)
    ends[:-2] = 0
    ends[-2], ends[-1] = T - 40, T
    a[:-40].zero_()
    b[-2].zero_()
    say("grouped product past 2^32 bytes")
    c = x.matmul_grouped(a, b, ends.cuda(), dtype=torch.bfloat16)           # 4.9 GB
    ref = rows.double() @ last.double()
    bound = 2 * U * (K + 8) * (rows.double().abs() @ last.double().abs()) + BF16 * ref.abs()
    within(host(c[-40:]), ref, bound, "last rows")
    assert bool((c[-1000:-40] == 0).all())
    del c, b
    say("quantize and norm past 2^32 bytes")
    q, s = x.quantize_fp8(a)
    check_e4m3(q[-40:], s[-40:], rows.double(), 1, 0.0, "last rows in 8 bits")
    n = x.rmsnorm(a, torch.ones(K, dtype=torch.bfloat16, device="cuda"))
    _, _, y = norm_reference(rows, torch.ones(K), None, 1e-6)
    within(host(n.out[-40:]), y, (BF16 + 2 * (K + 16) * U) * y.abs(), "last rows normed")


# ------------------------------------------------------ the native entries


def test_native_and_python_paths_of_the_operators_agree(monkeypatch):
    """The plain calls go through the native module; without it the same library is called from Python."""
    v = normal(1, 40, 264).bfloat16().cuda()
    w = torch.ones(264, dtype=torch.bfloat16, device="cuda")
    wq, ws = x.quantize_fp8(normal(2, 130, 264).float().cuda(), block_rows=128)
    fam = normal(3, 3, 264, 72).bfloat16().cuda()
    famq = wq.view(torch.uint8).expand(3, 130, 264).contiguous().view(torch.float8_e4m3fn)
    fams = ws.expand(3, *ws.shape).contiguous()
    ends = torch.tensor([7, 30, 38], dtype=torch.int32, device="cuda")
    out = torch.empty(40, 130, dtype=torch.bfloat16, device="cuda")

    def calls():
        n = x.rmsnorm(v, w, v, eps=1e-5, quantize=True)
        m = x.rmsnorm(v, w.float())
        assert type(n) is x.RmsNorm and m.scale is None and m.residual is v
        yield from (n.out.float(), n.scale, n.residual, n.rstd, m.out, m.rstd)
        yield from x.rmsnorm_backward(v, n.residual, w, n.rstd, v)
        q, s = x.quantize_fp8(v)
        yield from (q.float(), s, x.matmul_fp8(q, s, wq, ws), x.matmul_fp8(q, s, wq, ws, relu=True, dtype=torch.bfloat16))
        assert x.matmul_fp8(q, s, wq, ws, out=out) is out
        yield out.clone()
        yield x.matmul_grouped(v, fam, ends, relu=True)
        yield x.matmul_grouped(v, fam.transpose(1, 2).contiguous(), ends, transpose_b=True, dtype=torch.bfloat16)
        yield x.matmul_grouped_wgrad(v, v[:, :80].contiguous(), ends, dtype=torch.bfloat16)
        yield x.matmul_grouped_fp8(q, s, famq, fams, ends)

    assert x._fast is not None
    native = [t.clone() for t in calls()]
    monkeypatch.setattr(x, "_fast", None)
    for a, b in zip(native, calls()):
        assert a.dtype == b.dtype and torch.equal(a, b)


def test_captured_in_a_graph():
    """Replays give what eager calls give, with new values in the same tensors."""
    v = normal(1, 33, 512).bfloat16().cuda()
    w = torch.ones(512, dtype=torch.bfloat16, device="cuda")
    wq, ws = x.quantize_fp8(normal(2, 200, 512).float().cuda(), block_rows=128)
    fam = normal(3, 4, 512, 96).bfloat16().cuda()
    ends = torch.tensor([3, 9, 9, 33], dtype=torch.int32, device="cuda")

    def chain():
        n = x.rmsnorm(v, w, v, quantize=True)
        dx, dw = x.rmsnorm_backward(v, n.residual, w, n.rstd)
        return [x.matmul_fp8(n.out, n.scale, wq, ws), x.matmul_grouped(n.residual, fam, ends),
                x.matmul_grouped_wgrad(v, n.residual, ends), dx, dw]

    chain()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = chain()
    for seed in range(4):
        v.copy_(normal(10 + seed, 33, 512).bfloat16())
        ends.copy_(torch.tensor([[3, 9, 9, 33], [0, 0, 33, 33], [8, 16, 24, 30], [33, 33, 33, 33]][seed], dtype=torch.int32))
        graph.replay()
        torch.cuda.synchronize()
        want = chain()
        for a, b in zip(captured, want):
            assert torch.equal(a, b)


def test_rmsnorm_of_rows_without_columns():
    """The mean of nothing is 0/0: rstd is NaN, whatever its memory held before."""
    for dtype in ("f32", "bf16"):
        for quantize in (False, True):
            xs, w = (as_type(torch.zeros(*s), dtype).cuda() for s in ((50, 0), (0,)))
            for value in (3.0, 7.0):
                junk = torch.full((50,), value, device="cuda")
                del junk
                n = x.rmsnorm(xs, w, xs, quantize=quantize)
                assert n.out.shape == n.residual.shape == (50, 0) and n.rstd.shape == (50,)
                assert bool(torch.isnan(n.rstd).all())
                dx, dw = x.rmsnorm_backward(xs, xs, w, n.rstd)
                assert dx.shape == (50, 0) and dw.shape == (0,)

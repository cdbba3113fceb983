"""The work of the 8-bit, grouped and normalisation operators whose time matters, as measurable cases.

A case is one pass through ``rmsnorm`` or ``rmsnorm_backward``, ``quantize_fp8``,
``matmul_fp8``, ``matmul_grouped`` (with its gradients) or ``matmul_grouped_fp8`` on device
tensors, as a program that runs a transformer block makes it.  ``listed`` holds
one case per kind of work, ``draw`` samples the same kinds over their whole
range of sizes.  With ``own`` the framework's operators run; without it their plain
forms, elementary torch operations in 32 bits, rounded once at the end.
"""
import math

import torch

own = False

BLOCK = 128          # values that share a scale along a row
MOST = 448.0         # largest e4m3 value
TINY = 2.0 ** -126   # least scale
EPS = 1e-6


def _norm(T, D, dtype="bf16", residual=True, quantize=False, name=None):
    c = {"op": "rmsnorm", "T": T, "D": D, "dtype": dtype, "residual": residual, "quantize": quantize}
    return dict(c, name=name) if name else c


def _norm_backward(T, D, dtype="bf16", residual=True, name=None):
    c = {"op": "rmsnorm_backward", "T": T, "D": D, "dtype": dtype, "residual": residual}
    return dict(c, name=name) if name else c


def _quantize(M, K, dtype="bf16", rows=1, name=None):
    c = {"op": "quantize_fp8", "M": M, "K": K, "dtype": dtype, "rows": rows}
    return dict(c, name=name) if name else c


def _fp8(M, N, K, out="bf16", relu=False, name=None):
    c = {"op": "matmul_fp8", "M": M, "N": N, "K": K, "out": out, "relu": relu}
    return dict(c, name=name) if name else c


def _grouped(kind, T, E, N, K, out="bf16", relu=False, name=None):
    c = {"op": "grouped_" + kind, "T": T, "E": E, "N": N, "K": K, "out": out, "relu": relu}
    return dict(c, name=name) if name else c


def listed():
    return [
        # One token of a served request enters a block: the residual is added,
        # the sum normed and written in 8 bits for the next product.  All latency.
        _norm(1, 4096, quantize=True, name="norm_fp8_1x4096"),
        # The same for a long prompt: a stream through HBM.
        _norm(8192, 4096, quantize=True, name="norm_fp8_8192x4096"),
        # A first norm in 32 bits, nothing added and nothing padded.
        _norm(1531, 1021, dtype="f32", residual=False, name="norm_f32_1531x1021"),
        # The gradient of a training batch, rows not a multiple of anything.
        _norm_backward(8191, 2048, name="norm_backward_8191x2048"),
        # Activations between two 8-bit products.
        _quantize(4096, 4096, name="quantize_rows_4096x4096"),
        # A weight matrix, 128x128 values a scale, its last blocks cut.
        _quantize(8192, 3001, rows=128, name="quantize_blocks_8192x3001"),
        # Seven requests that each generate a token: the product streams its weights.
        _fp8(7, 4096, 4096, name="fp8_7x4096x4096"),
        # A chunk of a prompt, its rows and its outputs not whole tiles.
        _fp8(1531, 2000, 4096, out="f32", name="fp8_1531x2000x4096"),
        # The headline product's sizes in 8 bits.
        _fp8(8192, 8192, 8192, name="fp8_8192x8192x8192"),
        # Training, forward: tokens sorted by expert, groups of very different sizes.
        _grouped("forward", 16384, 16, 2048, 1024, relu=True, name="grouped_16384_e16_1024to2048"),
        # Training, backward of the same layer: its inputs' and its weights' gradients.
        _grouped("backward", 16384, 16, 2048, 1024, name="grouped_backward_16384_e16"),
        # Serving: 100 routed rows over 32 experts in 8 bits, a few rows each, some none.
        _grouped("fp8", 100, 32, 1024, 4096, name="grouped_fp8_100_e32_4096to1024"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng, lo, hi, step):
    """A layer's width: a multiple of ``step`` in four draws of five, else any number."""
    v = _log(rng, lo, hi)
    return max(step, v // step * step) if rng.random() < 0.8 else v


def draw(rng):
    kind = rng.choice(["rmsnorm", "rmsnorm", "backward", "quantize", "fp8", "fp8", "fp8",
                       "g_forward", "g_backward", "g_fp8"])
    dtype = "f32" if rng.random() < 0.25 else "bf16"
    out = "f32" if rng.random() < 0.3 else "bf16"
    relu = rng.random() < 0.3
    if kind == "rmsnorm":
        return _norm(_log(rng, 1, 16384), _width(rng, 512, 8192, 64), dtype, rng.random() < 0.75,
                     rng.random() < 0.6)
    if kind == "backward":
        return _norm_backward(_log(rng, 16, 16384), _width(rng, 512, 8192, 64), dtype, rng.random() < 0.75)
    if kind == "quantize":
        rows = rng.choice([1, 1, 128])
        return _quantize(_log(rng, 1 if rows == 1 else 512, 8192), _width(rng, 512, 8192, 128), dtype, rows)
    if kind == "fp8":
        # from single tokens to the largest prompts
        return _fp8(_log(rng, 1, 8192), _width(rng, 512, 8192, 64), _width(rng, 512, 8192, 128), out, relu)
    E = _log(rng, 4, 64)
    if kind == "g_fp8":
        return _grouped("fp8", _log(rng, 8, 8192), E, _width(rng, 512, 4096, 64), _width(rng, 512, 4096, 128),
                        out, relu)
    if kind == "g_forward":
        return _grouped("forward", _log(rng, 8, 16384), E, _width(rng, 512, 4096, 64),
                        _width(rng, 512, 4096, 64), out, relu)
    return _grouped("backward", _log(rng, 256, 16384), E, _width(rng, 512, 4096, 64),
                    _width(rng, 512, 4096, 64))


# ---------------------------------------------------------------- inputs


def _dt(name):
    return torch.float32 if name == "f32" else torch.bfloat16


def _normal(g, *shape):
    return torch.randn(*shape, device="cuda", generator=g)


def _activations(g, rows, cols):
    """Rows of a residual stream: most channels about 1, a few much larger."""
    channel = torch.exp(0.5 * _normal(g, cols)) * (1 + 20 * (torch.rand(cols, device="cuda", generator=g) < 0.01))
    return _normal(g, rows, cols) * channel


def _blocks(x, rows):
    """``x`` [..., M, K] as e4m3 values and a scale for each ``rows`` x 128 block."""
    *lead, M, K = x.shape
    mb, kb = -(-M // rows), -(-K // BLOCK)
    p = torch.nn.functional.pad(x, (0, kb * BLOCK - K, 0, mb * rows - M)).view(*lead, mb, rows, kb, BLOCK)
    s = (p.abs().amax((-3, -1)) / MOST).clamp_min(TINY)
    q = (p / s[..., :, None, :, None]).view(*lead, mb * rows, kb * BLOCK)[..., :M, :K]
    return q.contiguous().to(torch.float8_e4m3fn), s.contiguous()


def _group_sizes(g, T, E):
    """Rows of each group: some experts are much more popular than others."""
    p = torch.softmax(0.8 * _normal(g, E), 0)
    which = torch.multinomial(p, T, replacement=True, generator=g)
    return torch.bincount(which, minlength=E)


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    s = dict(case)
    op = case["op"]
    if op in ("rmsnorm", "rmsnorm_backward"):
        T, D, dt = case["T"], case["D"], _dt(case["dtype"])
        s["x"] = _activations(g, T, D).to(dt)
        s["weight"] = (1 + 0.2 * _normal(g, D)).to(dt)
        s["r"] = (2 * _activations(g, T, D)).to(dt) if case["residual"] else None
        if op == "rmsnorm_backward":
            s["dy"] = (0.01 * _normal(g, T, D)).to(dt)
            s["r"] = (0.01 * _normal(g, T, D)).to(dt) if case["residual"] else None
            s["rstd"] = torch.rsqrt(s["x"].float().square().mean(1) + EPS)
    elif op == "quantize_fp8":
        s["x"] = _activations(g, case["M"], case["K"]).to(_dt(case["dtype"]))
    elif op == "matmul_fp8":
        s["a"], s["a_scale"] = _blocks(_activations(g, case["M"], case["K"]), 1)
        s["b"], s["b_scale"] = _blocks(_normal(g, case["N"], case["K"]) / math.sqrt(case["K"]), 128)
    else:
        T, E, N, K = case["T"], case["E"], case["N"], case["K"]
        sizes = _group_sizes(g, T, E)
        s["ends"] = torch.cumsum(sizes, 0).to(torch.int32)
        s["most"] = int(sizes.max())
        if op == "grouped_fp8":
            s["a"], s["a_scale"] = _blocks(_activations(g, T, K), 1)
            s["b"], s["b_scale"] = _blocks(_normal(g, E, N, K) / math.sqrt(K), 128)
        else:
            s["a"] = _activations(g, T, K).bfloat16()
            s["b"] = (_normal(g, E, K, N) / math.sqrt(K)).bfloat16()
            s["dy"] = (0.01 * _normal(g, T, N)).bfloat16() if op == "grouped_backward" else None
    return s


# ----------------------------------------------------------- plain forms


def _plain_quantized(y, rows):
    """e4m3 values and scales of ``y`` in 32 bits; what is not finite becomes NaN."""
    M, K = y.shape
    mb, kb = -(-M // rows), -(-K // BLOCK)
    p = torch.nn.functional.pad(y, (0, kb * BLOCK - K, 0, mb * rows - M)).view(mb, rows, kb, BLOCK)
    fine = p.isfinite()
    s = (torch.where(fine, p.abs(), 0.0).amax((1, 3)) / MOST).clamp_min(TINY)
    q = torch.where(fine, p / s[:, None, :, None], math.nan)
    return q.view(mb * rows, kb * BLOCK)[:M, :K].contiguous().to(torch.float8_e4m3fn), s


def _plain_values(q, s, rows):
    """What e4m3 values and their scales stand for, in 32 bits."""
    M, K = q.shape[-2:]
    s = s.repeat_interleave(rows, -2)[..., :M, :] if rows > 1 else s
    return q.float() * s.repeat_interleave(BLOCK, -1)[..., :K]


def _padded(s, rows):
    """``rows`` [T, C] in 32 bits as [E, most, C], zeros past each group's end,
    and the place of each row there."""
    ends = s["ends"].long()
    t = torch.arange(rows.shape[0], device="cuda")
    group = torch.searchsorted(ends, t, right=True)
    start = torch.cat([ends.new_zeros(1), ends[:-1]])
    place = group * s["most"] + t - start[group]
    p = torch.zeros(s["E"] * s["most"], rows.shape[1], device="cuda")
    p[place] = rows.float()
    return p.view(s["E"], s["most"], -1), place


def _plain(s):
    op = s["op"]
    if op == "rmsnorm":
        h = s["x"].float() if s["r"] is None else s["x"].float() + s["r"].float()
        rstd = torch.rsqrt(h.square().mean(1) + EPS)
        y = h * rstd[:, None] * s["weight"].float()
        total = None if s["r"] is None else h.to(s["x"].dtype)
        if s["quantize"]:
            q, scale = _plain_quantized(y, 1)
            return {"out": q, "scale": scale, "residual": total, "rstd": rstd}
        return {"out": y.to(s["x"].dtype), "residual": total, "rstd": rstd}
    if op == "rmsnorm_backward":
        dy, xh = s["dy"].float(), s["x"].float() * s["rstd"][:, None]
        g = dy * s["weight"].float()
        dx = s["rstd"][:, None] * (g - xh * (g * xh).mean(1, keepdim=True))
        dx = dx if s["r"] is None else dx + s["r"].float()
        return {"dx": dx.to(s["x"].dtype), "dweight": (dy * xh).sum(0)}
    if op == "quantize_fp8":
        q, scale = _plain_quantized(s["x"].float(), s["rows"])
        return {"q": q, "scale": scale}
    if op == "matmul_fp8":
        y = _plain_values(s["a"], s["a_scale"], 1) @ _plain_values(s["b"], s["b_scale"], 128).t()
        return (y.relu() if s["relu"] else y).to(_dt(s["out"]))
    if op == "grouped_backward":
        dy, place = _padded(s, s["dy"])
        a, _ = _padded(s, s["a"])
        dx = torch.bmm(dy, s["b"].float().transpose(1, 2).contiguous())
        dw = torch.bmm(a.transpose(1, 2).contiguous(), dy)
        return {"dx": dx.view(-1, dx.shape[2])[place].to(_dt(s["out"])), "dweight": dw}
    if op == "grouped_fp8":
        a, place = _padded(s, _plain_values(s["a"], s["a_scale"], 1))
        b = _plain_values(s["b"], s["b_scale"], 128).transpose(1, 2).contiguous()
    else:
        a, place = _padded(s, s["a"])
        b = s["b"].float()
    y = torch.bmm(a, b)
    y = y.view(-1, y.shape[2])[place]
    return (y.relu() if s["relu"] else y).to(_dt(s["out"]))


# ------------------------------------------------------------- the passes


def _own(s):
    import paper_2512_16512_amd as xtc
    op = s["op"]
    if op == "rmsnorm":
        n = xtc.rmsnorm(s["x"], s["weight"], residual=s["r"], eps=EPS, quantize=s["quantize"])
        total = None if s["r"] is None else n.residual
        if s["quantize"]:
            return {"out": n.out, "scale": n.scale, "residual": total, "rstd": n.rstd}
        return {"out": n.out, "residual": total, "rstd": n.rstd}
    if op == "rmsnorm_backward":
        dx, dw = xtc.rmsnorm_backward(s["dy"], s["x"], s["weight"], s["rstd"], dresidual=s["r"])
        return {"dx": dx, "dweight": dw}
    if op == "quantize_fp8":
        q, scale = xtc.quantize_fp8(s["x"], block_rows=s["rows"])
        return {"q": q, "scale": scale}
    if op == "matmul_fp8":
        return xtc.matmul_fp8(s["a"], s["a_scale"], s["b"], s["b_scale"], relu=s["relu"], dtype=_dt(s["out"]))
    if op == "grouped_backward":
        return {"dx": xtc.matmul_grouped(s["dy"], s["b"], s["ends"], transpose_b=True, dtype=_dt(s["out"])),
                "dweight": xtc.matmul_grouped_wgrad(s["a"], s["dy"], s["ends"])}
    if op == "grouped_fp8":
        return xtc.matmul_grouped_fp8(s["a"], s["a_scale"], s["b"], s["b_scale"], s["ends"], relu=s["relu"],
                                      dtype=_dt(s["out"]))
    return xtc.matmul_grouped(s["a"], s["b"], s["ends"], relu=s["relu"], dtype=_dt(s["out"]))


def run(state):
    return _own(state) if own else _plain(state)


def work(case):
    op = case["op"]
    if op in ("rmsnorm", "rmsnorm_backward"):
        T, D, e = case["T"], case["D"], 4 if case["dtype"] == "f32" else 2
        if op == "rmsnorm_backward":
            arrays = 4 if case["residual"] else 3                   # dy, x, dx (and the sum's own gradient)
            return {"bytes": T * D * e * arrays + D * (e + 4) + T * 4, "flops": 10 * T * D}
        y = T * D + T * -(-D // BLOCK) * 4 if case["quantize"] else T * D * e
        return {"bytes": T * D * e * (3 if case["residual"] else 1) + y + D * e + T * 4, "flops": 6 * T * D}
    if op == "quantize_fp8":
        M, K, e = case["M"], case["K"], 4 if case["dtype"] == "f32" else 2
        return {"bytes": M * K * (e + 1) + -(-M // case["rows"]) * -(-K // BLOCK) * 4, "flops": 3 * M * K}
    N, K, o = case["N"], case["K"], 4 if case["out"] == "f32" else 2
    kb = -(-K // BLOCK)
    if op == "matmul_fp8":
        M = case["M"]
        return {"bytes": M * K + N * K + 4 * kb * (M + -(-N // 128)) + M * N * o, "flops": 2 * M * N * K}
    T, E = case["T"], min(case["E"], case["T"])                    # a group without rows reads no weights
    if op == "grouped_fp8":
        return {"bytes": T * K + E * N * K + 4 * kb * (T + E * -(-N // 128)) + T * N * o, "flops": 2 * T * N * K}
    if op == "grouped_forward":
        return {"bytes": 2 * (T * K + E * N * K) + T * N * o, "flops": 2 * T * N * K}
    return {"bytes": 2 * (T * N + T * K + E * N * K) + T * K * o + 4 * case["E"] * N * K, "flops": 4 * T * N * K}


# ---------------------------------------------------------------- 64 bits


def _stands_for(q, scale, rows):
    """The 64-bit values of a block-scaled matrix."""
    k = torch.arange(q.shape[1], device="cuda") // BLOCK
    m = torch.arange(q.shape[0], device="cuda") // rows
    return q.double() * scale.double()[m][:, k]


def _scaled(y, rows):
    """64-bit values over their block's scale (before they are rounded to 8 bits), and the scales."""
    M, K = y.shape
    mb, kb = -(-M // rows), -(-K // BLOCK)
    scale = torch.empty(mb, kb, dtype=torch.float64, device="cuda")
    out = torch.empty_like(y)
    for c in range(kb):
        cut = y[:, c * BLOCK:(c + 1) * BLOCK]
        row = cut.abs().max(1).values
        top = torch.zeros(mb * rows, dtype=torch.float64, device="cuda")
        top[:M] = row
        scale[:, c] = torch.clamp(top.reshape(mb, rows).max(1).values / MOST, min=TINY)
        out[:, c * BLOCK:(c + 1) * BLOCK] = cut / scale[:, c].repeat_interleave(rows)[:M, None]
    return out, scale


def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op == "rmsnorm":
        h = s["x"].double()
        if s["r"] is not None:
            h = h + s["r"].double()
        rstd = 1 / torch.sqrt((h * h).sum(1) / case["D"] + EPS)
        y = s["weight"].double() * (h * rstd[:, None])
        total = None if s["r"] is None else h
        if case["quantize"]:
            q, scale = _scaled(y, 1)
            return {"out": q, "scale": scale, "residual": total, "rstd": rstd}
        return {"out": y, "residual": total, "rstd": rstd}
    if op == "rmsnorm_backward":
        dy, x, w, r = s["dy"].double(), s["x"].double(), s["weight"].double(), s["rstd"].double()[:, None]
        along = (dy * w * x).sum(1, keepdim=True) / case["D"]       # d rstd / d x is -rstd^3 x / D
        dx = r * dy * w - r ** 3 * x * along
        if s["r"] is not None:
            dx = dx + s["r"].double()
        return {"dx": dx, "dweight": (dy * x * r).sum(0)}
    if op == "quantize_fp8":
        q, scale = _scaled(s["x"].double(), case["rows"])
        return {"q": q, "scale": scale}
    if op == "matmul_fp8":
        y = _stands_for(s["a"], s["a_scale"], 1) @ _stands_for(s["b"], s["b_scale"], 128).t().contiguous()
        return torch.where(y < 0, 0.0, y) if case["relu"] else y
    ends = [0] + s["ends"].tolist()
    T, E, N, K = case["T"], case["E"], case["N"], case["K"]
    if op == "grouped_backward":
        dx = torch.zeros(T, K, dtype=torch.float64, device="cuda")
        dw = torch.zeros(E, K, N, dtype=torch.float64, device="cuda")
        for e in range(E):
            i, j = ends[e], ends[e + 1]
            if j > i:
                dy = s["dy"][i:j].double()
                dx[i:j] = dy @ s["b"][e].double().t().contiguous()
                dw[e] = s["a"][i:j].double().t().contiguous() @ dy
        return {"dx": dx, "dweight": dw}
    y = torch.zeros(T, N, dtype=torch.float64, device="cuda")
    for e in range(E):
        i, j = ends[e], ends[e + 1]
        if j <= i:
            continue
        if op == "grouped_fp8":
            a = _stands_for(s["a"][i:j], s["a_scale"][i:j], 1)
            b = _stands_for(s["b"][e], s["b_scale"][e], 128).t().contiguous()
        else:
            a, b = s["a"][i:j].double(), s["b"][e].double()
        y[i:j] = a @ b
    return torch.where(y < 0, 0.0, y) if case["relu"] else y

"""The work of the layer norm, linear, routing and combining operators whose time matters, as measurable cases.

A case is one pass through ``layernorm`` or ``layernorm_backward``, ``linear`` or its
gradients (``linear_wgrad``, ``activation_backward``), ``route_experts`` or
``route_experts_backward``, ``combine_experts`` or ``combine_experts_backward`` on device
tensors, as a program that runs the feed-forward half of a transformer block makes it.
``listed`` holds one case per kind of work, ``draw`` samples the same kinds over their
whole range of sizes.  With ``own`` the framework's operators run; without it their plain
forms, elementary torch operations in 32 bits, rounded once at the end.
"""
import math

import torch

own = False

BLOCK = 128          # values that share a scale along a row
MOST = 448.0         # largest e4m3 value
TINY = 2.0 ** -126   # least scale
EPS = 1e-5
LARGEST = 8192 * 4096 * 4096   # products of the largest listed layer


def _norm(T, D, dtype="bf16", residual=True, quantize=False, name=None):
    c = {"op": "layernorm", "T": T, "D": D, "dtype": dtype, "residual": residual, "quantize": quantize}
    return dict(c, name=name) if name else c


def _norm_backward(T, D, dtype="bf16", residual=True, name=None):
    c = {"op": "layernorm_backward", "T": T, "D": D, "dtype": dtype, "residual": residual}
    return dict(c, name=name) if name else c


def _linear(T, K, N, act="none", residual=False, turned=False, keep=False, out="bf16", name=None):
    c = {"op": "linear", "T": T, "K": K, "N": N, "act": act, "residual": residual, "turned": turned, "keep": keep,
         "out": out}
    return dict(c, name=name) if name else c


def _linear_grads(T, K, N, turned=False, name=None):
    c = {"op": "linear_grads", "T": T, "K": K, "N": N, "turned": turned}
    return dict(c, name=name) if name else c


def _activation(T, N, act, name=None):
    c = {"op": "activation_backward", "T": T, "N": N, "act": act}
    return dict(c, name=name) if name else c


def _route(T, E, top, dtype="f32", masked=False, backward=False, name=None):
    c = {"op": "route_backward" if backward else "route", "T": T, "E": E, "top": top, "dtype": dtype, "masked": masked}
    return dict(c, name=name) if name else c


def _combine(T, top, D, dtype="bf16", residual=False, backward=False, name=None):
    c = {"op": "combine_backward" if backward else "combine", "T": T, "top": top, "D": D, "dtype": dtype,
         "residual": residual}
    return dict(c, name=name) if name else c


def listed():
    return [
        # A long prompt enters a block: the residual is added and the sum normed, a stream through HBM.
        _norm(8192, 4096, name="layernorm_8192x4096"),
        # The gradient of a training batch, rows not a multiple of anything.
        _norm_backward(8191, 2048, name="layernorm_backward_8191x2048"),
        # One token of a served request leaves the attention: its projection, bias and
        # residual.  The weights are read once.
        _linear(1, 4096, 4096, residual=True, name="linear_1x4096to4096"),
        # A chunk of a prompt, its rows and its outputs not whole tiles, weights a row an output.
        _linear(1531, 4096, 2000, act="silu", turned=True, out="f32", name="linear_1531x4096to2000"),
        # Training, forward: the first layer of a feed-forward block, what its activation took kept.
        _linear(8192, 4096, 4096, act="gelu_tanh", keep=True, name="linear_8192x4096to4096"),
        # Training, backward of a narrower layer: its inputs' and its weights' gradients.
        _linear_grads(16384, 1024, 2048, name="linear_grads_16384x1024to2048"),
        # The activation's and the bias's gradient.
        _activation(8192, 4096, "gelu_tanh", name="activation_backward_8192x4096"),
        # One token of a served request chooses its experts.  All latency.
        _route(1, 64, 8, name="route_1_e64"),
        # A training batch, some of it padding, over many experts; scores of a bf16 product have ties.
        _route(16383, 128, 8, dtype="bf16", masked=True, name="route_16383_e128"),
        # The router's gradient, the balance loss's part in it.
        _route(16384, 64, 6, backward=True, name="route_backward_16384_e64"),
        # The experts' rows come back to their tokens.
        _combine(4096, 8, 2048, residual=True, name="combine_4096_top8"),
        # The gradient of that: each expert's rows' and the weights'.
        _combine(4095, 8, 2048, backward=True, name="combine_backward_4095_top8"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng, lo, hi, step):
    """A layer's width: a multiple of ``step`` in four draws of five, else any number."""
    v = _log(rng, lo, hi)
    return max(step, v // step * step) if rng.random() < 0.8 else v


def draw(rng):
    kind = rng.choice(["norm", "norm_backward", "linear", "linear", "linear", "linear", "grads", "grads", "activation",
                       "route", "route", "route_backward", "combine", "combine_backward"])
    dtype = "f32" if rng.random() < 0.25 else "bf16"
    act = rng.choice(["none", "relu", "gelu", "gelu_tanh", "silu"])
    if kind == "norm":
        return _norm(_log(rng, 1, 8192), _width(rng, 512, 4096, 64), dtype, rng.random() < 0.6, rng.random() < 0.3)
    if kind == "norm_backward":
        return _norm_backward(_log(rng, 16, 8192), _width(rng, 512, 4096, 64), dtype, rng.random() < 0.6)
    if kind == "activation":
        return _activation(_log(rng, 16, 8192), _width(rng, 512, 4096, 64), "silu" if act == "none" else act)
    if kind in ("linear", "grads"):
        # from single tokens to the largest batches, no layer larger than the listed ones
        T = _log(rng, 1 if kind == "linear" else 64, 8192)
        K, N = _width(rng, 512, 8192, 64), _width(rng, 512, 8192, 64)
        while T * K * N > (LARGEST if kind == "linear" else LARGEST // 2):
            K, N = (max(512, K // 2), N) if K > N else (K, max(512, N // 2))
        if kind == "grads":
            return _linear_grads(T, K, N, rng.random() < 0.5)
        return _linear(T, K, N, act, rng.random() < 0.5, rng.random() < 0.5, rng.random() < 0.3, dtype)
    if kind in ("route", "route_backward"):
        E = rng.choice([8, 16, 32, 64, 128, 256, 60, 200, 7])
        top = min(E, rng.choice([1, 2, 2, 4, 6, 8, 8]))
        return _route(_log(rng, 1, 16384), E, top, "bf16" if rng.random() < 0.4 else "f32", rng.random() < 0.4,
                      kind == "route_backward")
    return _combine(_log(rng, 1, 4096), rng.choice([1, 2, 4, 6, 8]), _width(rng, 512, 2048, 64), dtype,
                    rng.random() < 0.5, kind == "combine_backward")


# ---------------------------------------------------------------- inputs


def _dt(name):
    return torch.float32 if name == "f32" else torch.bfloat16


def _act_name(case):
    return None if case["act"] == "none" else case["act"]


def _normal(g, *shape):
    return torch.randn(*shape, device="cuda", generator=g)


def _activations(g, rows, cols):
    """Rows of a residual stream: most channels about 1 and off zero, a few much larger."""
    channel = torch.exp(0.5 * _normal(g, cols)) * (1 + 20 * (torch.rand(cols, device="cuda", generator=g) < 0.01))
    return (_normal(g, rows, cols) + 0.3 * _normal(g, cols)) * channel


def _scores(g, T, E):
    """A router's scores: some experts are much more popular than others."""
    return _normal(g, T, E) + 0.8 * _normal(g, E)


def _chosen(scores, top, mask):
    """What the router would hand its gradient: experts, their weights and counts."""
    E = scores.shape[1]
    v, e = torch.sort(scores.float(), dim=1, descending=True, stable=True)
    p = torch.softmax(v[:, :top], 1)
    e = e[:, :top].to(torch.int32)
    if mask is not None:
        e, p = torch.where(mask[:, None], e, -1), torch.where(mask[:, None], p, 0.0)
    counts = torch.zeros(E + 1, device="cuda").index_add_(0, torch.where(e < 0, E, e).flatten().long(),
                                                          torch.ones(e.numel(), device="cuda"))
    return e.contiguous(), p.contiguous(), counts[:E].to(torch.int32)


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    s = dict(case)
    op = case["op"]
    if op in ("layernorm", "layernorm_backward"):
        T, D, dt = case["T"], case["D"], _dt(case["dtype"])
        s["x"] = _activations(g, T, D).to(dt)
        s["weight"] = (1 + 0.2 * _normal(g, D)).to(dt)
        s["bias"] = (0.1 * _normal(g, D)).to(dt)
        s["r"] = (2 * _activations(g, T, D)).to(dt) if case["residual"] else None
        if op == "layernorm_backward":
            s["dy"] = (0.01 * _normal(g, T, D)).to(dt)
            s["r"] = (0.01 * _normal(g, T, D)).to(dt) if case["residual"] else None
            x = s["x"].float()
            s["mean"] = x.mean(1)
            s["rstd"] = torch.rsqrt((x - s["mean"][:, None]).square().mean(1) + EPS)
    elif op in ("linear", "linear_grads"):
        T, K, N = case["T"], case["K"], case["N"]
        s["a"] = _normal(g, T, K).bfloat16()
        b = _normal(g, N, K) if case["turned"] else _normal(g, K, N)
        s["b"] = (b / math.sqrt(K)).bfloat16()
        if op == "linear":
            s["bias"] = (0.2 * _normal(g, N)).bfloat16()
            s["r"] = (2 * _normal(g, T, N)).bfloat16() if case["residual"] else None
        else:
            s["dz"] = (0.01 * _normal(g, T, N)).bfloat16()
    elif op == "activation_backward":
        s["z"] = (1.5 * _normal(g, case["T"], case["N"])).bfloat16()
        s["dy"] = (0.01 * _normal(g, case["T"], case["N"])).bfloat16()
    elif op in ("route", "route_backward"):
        T, E, top = case["T"], case["E"], case["top"]
        s["scores"] = _scores(g, T, E).to(_dt(case["dtype"]))
        s["mask"] = torch.rand(T, device="cuda", generator=g) < 0.9 if case["masked"] else None
        if op == "route_backward":
            s["expert"], s["p"], s["counts"] = _chosen(s["scores"], top, s["mask"])
            s["dp"] = 0.1 * _normal(g, T, top)
            s["dloss"] = 0.01
    else:
        T, top, D, dt = case["T"], case["top"], case["D"], _dt(case["dtype"])
        order = torch.randperm(T * top, device="cuda", generator=g)
        s["row"] = order.view(T, top).to(torch.int32)
        s["token"] = torch.empty_like(order)
        s["token"][order] = torch.arange(T * top, device="cuda") // top
        s["token"] = s["token"].to(torch.int32)
        s["rows"] = _normal(g, T * top, D).to(dt)
        s["p"] = torch.softmax(_normal(g, T, top), 1)
        if op == "combine_backward":
            s["dout"] = (0.01 * _normal(g, T, D)).to(dt)
        else:
            s["r"] = (2 * _normal(g, T, D)).to(dt) if case["residual"] else None
    return s


# ----------------------------------------------------------- plain forms


def _plain_quantized(y):
    """e4m3 values of ``y`` in 32 bits and a scale for each 128 of a row."""
    M, K = y.shape
    kb = -(-K // BLOCK)
    p = torch.nn.functional.pad(y, (0, kb * BLOCK - K)).view(M, kb, BLOCK)
    s = (p.abs().amax(2) / MOST).clamp_min(TINY)
    return (p / s[:, :, None]).view(M, kb * BLOCK)[:, :K].contiguous().to(torch.float8_e4m3fn), s


def _plain_act(z, act):
    if act == "relu":
        return torch.where(z < 0, 0.0, z)
    if act == "gelu":
        return 0.5 * z * (1 + torch.erf(z * math.sqrt(0.5)))
    if act == "gelu_tanh":
        return 0.5 * z * (1 + torch.tanh(math.sqrt(2 / math.pi) * (z + 0.044715 * z * z * z)))
    if act == "silu":
        return z / (1 + torch.exp(-z))
    return z


def _plain_slope(z, act):
    if act == "relu":
        return (z > 0).to(z.dtype)
    if act == "gelu":
        return 0.5 * (1 + torch.erf(z * math.sqrt(0.5))) + z * torch.exp(-0.5 * z * z) / math.sqrt(2 * math.pi)
    if act == "gelu_tanh":
        c = math.sqrt(2 / math.pi)
        t = torch.tanh(c * (z + 0.044715 * z * z * z))
        return 0.5 * (1 + t) + 0.5 * z * (1 - t * t) * c * (1 + 3 * 0.044715 * z * z)
    if act == "silu":
        q = 1 / (1 + torch.exp(-z))
        return q * (1 + z * (1 - q))
    return torch.ones_like(z)


def _plain_softmax(v):
    e = torch.exp(v - v.amax(1, keepdim=True))
    return e / e.sum(1, keepdim=True)


def _plain(s):
    op = s["op"]
    if op == "layernorm":
        h = s["x"].float() if s["r"] is None else s["x"].float() + s["r"].float()
        mean = h.mean(1)
        d = h - mean[:, None]
        rstd = torch.rsqrt(d.square().mean(1) + EPS)
        y = d * rstd[:, None] * s["weight"].float() + s["bias"].float()
        res = {"residual": None if s["r"] is None else h.to(s["x"].dtype), "mean": mean, "rstd": rstd}
        if s["quantize"]:
            q, scale = _plain_quantized(y)
            return dict(res, out=q, scale=scale)
        return dict(res, out=y.to(s["x"].dtype))
    if op == "layernorm_backward":
        dy, xh = s["dy"].float(), (s["x"].float() - s["mean"][:, None]) * s["rstd"][:, None]
        g = dy * s["weight"].float()
        dx = s["rstd"][:, None] * (g - g.mean(1, keepdim=True) - xh * (g * xh).mean(1, keepdim=True))
        dx = dx if s["r"] is None else dx + s["r"].float()
        return {"dx": dx.to(s["x"].dtype), "dweight": (dy * xh).sum(0), "dbias": dy.sum(0)}
    if op == "linear":
        b = s["b"].float()
        z = s["a"].float() @ (b.t() if s["turned"] else b) + s["bias"].float()
        y = _plain_act(z, s["act"])
        y = y if s["r"] is None else y + s["r"].float()
        return {"out": y.to(_dt(s["out"])), "z": z.to(_dt(s["out"])) if s["keep"] else None}
    if op == "linear_grads":
        dz, a, b = s["dz"].float(), s["a"].float(), s["b"].float()
        return {"da": (dz @ (b if s["turned"] else b.t())).bfloat16(), "db": dz.t() @ a if s["turned"] else a.t() @ dz}
    if op == "activation_backward":
        dz = s["dy"].float() * _plain_slope(s["z"].float(), s["act"])
        return {"dz": dz.bfloat16(), "dbias": dz.sum(0)}
    if op == "route":
        v = s["scores"].float()
        T, E = v.shape
        top, mask = s["top"], s["mask"]
        best, expert = torch.sort(v, dim=1, descending=True, stable=True)
        p, expert, q = _plain_softmax(best[:, :top]), expert[:, :top], _plain_softmax(v)
        n = torch.full((), float(T), device="cuda")
        if mask is not None:
            expert = torch.where(mask[:, None], expert, E)
            p, q = torch.where(mask[:, None], p, 0.0), torch.where(mask[:, None], q, 0.0)
            n = mask.float().sum().clamp_min(1)
        by, order = torch.sort(expert.flatten(), stable=True)
        ends = torch.searchsorted(by, torch.arange(E, device="cuda"), right=True, out_int32=True)
        counts = torch.diff(ends, prepend=ends.new_zeros(1))
        row = torch.empty_like(order)
        row[order] = torch.arange(T * top, device="cuda")
        loss = E / (top * n * n) * (counts.float() * q.sum(0)).sum()
        out = expert < E
        return {"expert": torch.where(out, expert, -1).int(), "p": p, "row": torch.where(out, row.view(T, top), -1).int(),
                "token": torch.where(by < E, order // top, -1).int(), "counts": counts, "ends": ends, "loss": loss}
    if op == "route_backward":
        v = s["scores"].float()
        T, E = v.shape
        there = s["expert"][:, :1] >= 0
        q, c = torch.where(there, _plain_softmax(v), 0.0), s["counts"].float()
        n = there.float().sum().clamp_min(1)
        d = s["dloss"] * E / (s["top"] * n * n) * q * (c - (c * q).sum(1, keepdim=True))
        chosen = s["p"] * (s["dp"] - (s["dp"] * s["p"]).sum(1, keepdim=True))
        return d.scatter_add(1, s["expert"].clamp_min(0).long(), chosen).to(s["scores"].dtype)
    if op == "combine":
        y = (s["rows"].float()[s["row"].long()] * s["p"][:, :, None]).sum(1)
        return (y if s["r"] is None else y + s["r"].float()).to(_dt(s["dtype"]))
    dout, row = s["dout"].float(), s["row"].long()
    drows = torch.empty_like(s["rows"])
    drows[row.flatten()] = (s["p"][:, :, None] * dout[:, None]).to(drows.dtype).flatten(0, 1)
    return {"drows": drows, "dp": (s["rows"].float()[row] * dout[:, None]).sum(2)}


# ------------------------------------------------------------- the passes


def _own(s):
    import paper_2512_16512_amd as xtc
    op = s["op"]
    if op == "layernorm":
        n = xtc.layernorm(s["x"], s["weight"], s["bias"], residual=s["r"], eps=EPS, quantize=s["quantize"])
        res = {"residual": None if s["r"] is None else n.residual, "mean": n.mean, "rstd": n.rstd, "out": n.out}
        return dict(res, scale=n.scale) if s["quantize"] else res
    if op == "layernorm_backward":
        dx, dw, db = xtc.layernorm_backward(s["dy"], s["x"], s["weight"], s["mean"], s["rstd"], dresidual=s["r"])
        return {"dx": dx, "dweight": dw, "dbias": db}
    if op == "linear":
        y = xtc.linear(s["a"], s["b"], bias=s["bias"], residual=s["r"], activation=_act_name(s),
                       transpose_b=s["turned"], keep=s["keep"], dtype=_dt(s["out"]))
        return {"out": y[0], "z": y[1]} if s["keep"] else {"out": y, "z": None}
    if op == "linear_grads":
        da = xtc.linear(s["dz"], s["b"], transpose_b=not s["turned"], dtype=torch.bfloat16)
        return {"da": da, "db": xtc.linear_wgrad(s["dz"], s["a"]) if s["turned"] else xtc.linear_wgrad(s["a"], s["dz"])}
    if op == "activation_backward":
        dz, db = xtc.activation_backward(s["dy"], s["z"], s["act"])
        return {"dz": dz, "dbias": db}
    if op == "route":
        r = xtc.route_experts(s["scores"], s["top"], mask=s["mask"])
        return {"expert": r.expert, "p": r.p, "row": r.row, "token": r.token, "counts": r.counts, "ends": r.ends,
                "loss": r.loss}
    if op == "route_backward":
        return xtc.route_experts_backward(s["dp"], s["scores"], s["expert"], s["p"], s["counts"], dloss=s["dloss"])
    if op == "combine":
        return xtc.combine_experts(s["rows"], s["row"], s["p"], residual=s["r"], dtype=_dt(s["dtype"]))
    drows, dp = xtc.combine_experts_backward(s["dout"], s["rows"], s["row"], s["token"], s["p"])
    return {"drows": drows, "dp": dp}


def run(state):
    return _own(state) if own else _plain(state)


def work(case):
    op = case["op"]
    if op in ("layernorm", "layernorm_backward"):
        T, D, e = case["T"], case["D"], 4 if case["dtype"] == "f32" else 2
        if op == "layernorm_backward":
            arrays = 4 if case["residual"] else 3                   # dy, x, dx (and the sum's own gradient)
            return {"bytes": T * D * e * arrays + D * (e + 8) + T * 8, "flops": 14 * T * D}
        y = T * D + T * -(-D // BLOCK) * 4 if case["quantize"] else T * D * e
        return {"bytes": T * D * e * (3 if case["residual"] else 1) + y + 2 * D * e + T * 8, "flops": 9 * T * D}
    if op == "linear":
        T, K, N, o = case["T"], case["K"], case["N"], 4 if case["out"] == "f32" else 2
        moved = 2 * (T * K + K * N + N) + T * N * (o * (2 if case["keep"] else 1) + (2 if case["residual"] else 0))
        return {"bytes": moved, "flops": 2 * T * N * K}
    if op == "linear_grads":
        T, K, N = case["T"], case["K"], case["N"]
        return {"bytes": 2 * (T * N + 2 * T * K + N * K) + 4 * N * K, "flops": 4 * T * N * K}
    if op == "activation_backward":
        T, N = case["T"], case["N"]
        return {"bytes": 6 * T * N + 4 * N, "flops": 20 * T * N}
    if op in ("route", "route_backward"):
        T, E, top, e = case["T"], case["E"], case["top"], 4 if case["dtype"] == "f32" else 2
        if op == "route_backward":
            return {"bytes": 2 * T * E * e + 12 * T * top + 4 * E, "flops": 8 * T * E}
        return {"bytes": T * E * e + 16 * T * top + 8 * E + (T if case["masked"] else 0), "flops": 6 * T * E}
    T, top, D, e = case["T"], case["top"], case["D"], 4 if case["dtype"] == "f32" else 2
    if op == "combine":
        return {"bytes": T * D * e * (top + (2 if case["residual"] else 1)) + 8 * T * top, "flops": 2 * T * top * D}
    return {"bytes": T * D * e * (2 * top + 1) + 16 * T * top, "flops": 3 * T * top * D}


# ---------------------------------------------------------------- 64 bits


def _turn(t):
    """The transpose, laid out by rows."""
    return t.t().contiguous()


def _normal_cdf(z):
    return torch.special.erfc(-z / math.sqrt(2)) / 2


def _function(z, act):
    """The activation of ``z`` and its derivative in 64 bits."""
    if act == "relu":
        return torch.clamp(z, min=0), (z > 0).double()
    if act == "gelu":
        cdf = _normal_cdf(z)
        return z * cdf, cdf + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    if act == "gelu_tanh":
        u = math.sqrt(8 / math.pi) * (z + 0.044715 * z ** 3)        # (1 + tanh(u / 2)) / 2 is the logistic of u
        q = torch.sigmoid(u)
        return z * q, q + z * q * torch.sigmoid(-u) * math.sqrt(8 / math.pi) * (1 + 0.134145 * z ** 2)
    if act == "silu":
        q = torch.sigmoid(z)
        return z * q, q + z * q * torch.sigmoid(-z)
    return z, torch.ones_like(z)


def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op == "layernorm":
        h = s["x"].double()
        if s["r"] is not None:
            h = h + s["r"].double()
        mean = h.sum(1) / case["D"]
        centred = h - mean[:, None]
        rstd = 1 / torch.sqrt((centred * centred).sum(1) / case["D"] + EPS)
        y = s["bias"].double() + s["weight"].double() * (centred * rstd[:, None])
        total = None if s["r"] is None else h
        if not case["quantize"]:
            return {"out": y, "residual": total, "mean": mean, "rstd": rstd}
        scale = torch.stack([c.abs().amax(1) / MOST for c in y.split(BLOCK, 1)], 1).clamp(min=TINY)
        each = scale[:, torch.arange(case["D"], device="cuda") // BLOCK]
        return {"out": y / each, "scale": scale, "residual": total, "mean": mean, "rstd": rstd}
    if op == "layernorm_backward":
        dy, w, r = s["dy"].double(), s["weight"].double(), s["rstd"].double()[:, None]
        d = s["x"].double() - s["mean"].double()[:, None]
        # d rstd / d x_i is -rstd^3 (x_i - mean) / D, d mean / d x_i is 1 / D
        g = r * dy * w
        dx = g - g.sum(1, keepdim=True) / case["D"] - r ** 3 * d * (dy * w * d).sum(1, keepdim=True) / case["D"]
        if s["r"] is not None:
            dx = dx + s["r"].double()
        return {"dx": dx, "dweight": (dy * d * r).sum(0), "dbias": dy.sum(0)}
    if op == "linear":
        b = s["b"].double()
        z = torch.addmm(s["bias"].double(), s["a"].double(), _turn(b) if case["turned"] else b)
        y = _function(z, case["act"])[0]
        if s["r"] is not None:
            y = s["r"].double() + y
        return {"out": y, "z": z if case["keep"] else None}
    if op == "linear_grads":
        dz, a, b = s["dz"].double(), s["a"].double(), s["b"].double()
        if case["turned"]:
            return {"da": torch.mm(dz, b), "db": torch.mm(_turn(dz), a)}
        return {"da": torch.mm(dz, _turn(b)), "db": torch.mm(_turn(a), dz)}
    if op == "activation_backward":
        dz = _function(s["z"].double(), case["act"])[1] * s["dy"].double()
        return {"dz": dz, "dbias": dz.sum(0)}
    if op in ("route", "route_backward"):
        T, E, top = case["T"], case["E"], case["top"]
        v = s["scores"].double()
        there = torch.ones(T, dtype=torch.bool, device="cuda") if s["mask"] is None else s["mask"]
        n = max(1, int(there.sum()))
        q = torch.exp(torch.log_softmax(v, 1)) * there[:, None]
        if op == "route_backward":
            c = s["counts"].double()
            ds = s["dloss"] * E / (top * n ** 2) * (c * q - q * torch.mv(q, c)[:, None])
            p, dp = s["p"].double(), s["dp"].double()
            for j in range(top):
                e = s["expert"][:, j].long()
                at = torch.nonzero(e >= 0)[:, 0]
                ds[at, e[at]] += (p[:, j] * dp[:, j] - p[:, j] * (p * dp).sum(1))[at]
            return ds
        # the experts in turn, the highest first; of equal scores the lowest index
        left, chosen = v.clone(), torch.empty(T, top, dtype=torch.long, device="cuda")
        index = torch.arange(E, device="cuda")
        for j in range(top):
            most = left.amax(1, keepdim=True)
            chosen[:, j] = torch.where(left == most, index, E).amin(1)
            left.scatter_(1, chosen[:, j:j + 1], -math.inf)
        p = torch.exp(torch.log_softmax(v.gather(1, chosen), 1)) * there[:, None]
        counts = torch.stack([((chosen == e) & there[:, None]).sum() for e in range(E)])
        loss = E / (top * n ** 2) * torch.dot(counts.double(), q.sum(0))
        return {"expert": None, "p": p, "row": None, "token": None, "counts": None, "ends": None, "loss": loss}
    p, rows, T = s["p"].double(), s["rows"].double(), case["T"]
    if op == "combine":
        y = torch.zeros(T, case["D"], dtype=torch.float64, device="cuda")
        if s["r"] is not None:
            y += s["r"].double()
        for j in range(case["top"]):
            y += p[:, j:j + 1] * rows[s["row"][:, j].long()]
        return y
    dout, token = s["dout"].double(), s["token"].long()
    weight = torch.empty(token.shape[0], dtype=torch.float64, device="cuda")
    weight[s["row"].flatten().long()] = p.flatten()
    each = (rows * dout[token]).sum(1)
    return {"drows": weight[:, None] * dout[token], "dp": each[s["row"].long()]}

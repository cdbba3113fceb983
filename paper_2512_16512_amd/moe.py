"""A mixture-of-experts block on the norm, 8-bit, grouped, linear and routing operators: one
step of serving in 8 bits and one of training in bfloat16, as a program would make them.

    h = x + residual,  y = rmsnorm(h),  scores = y @ router.T
    out[t] = sum over t's top experts e of  p[t, e] * relu(y[t] @ w1[e]) @ w2[e]

With a bias for the norm it is a layer norm.  The training step can train the router too (through the
weights p and a balance loss) and can have an expert that every token passes, a dense pair of layers with
biases and an activation:

    out[t] += act(y[t] @ v1 + c1) @ v2 + c2

``python -m paper_2512_16512_amd.moe`` runs these on random weights and prints what a step takes.
Copying the rows to their experts (an indexing) is torch's.
"""
from __future__ import annotations

import argparse
import time
from collections import namedtuple

import torch

from . import (Routing, activation_backward, combine_experts, combine_experts_backward, layernorm, layernorm_backward,
               linear, linear_wgrad, matmul_fp8, matmul_grouped, matmul_grouped_fp8, matmul_grouped_wgrad, quantize_fp8,
               rmsnorm, rmsnorm_backward, route_experts, route_experts_backward)

MOST_EXPERTS, MOST_CHOSEN = 1024, 16      # what route_experts takes


def _fits(t):
    """Whether the operators take a matrix of values as it is: rows of neighbouring values that do not overlap."""
    rows, cols = t.shape
    return (t.is_cuda and t.dtype in (torch.float32, torch.bfloat16) and (cols <= 1 or t.stride(1) == 1) and
            (rows <= 1 or t.stride(0) >= max(cols, 1)))


def _watched(t):
    """Whether torch follows what happens to ``t``, which the library's calls do not show it: for a gradient, a tangent, a
    trace or a transformation."""
    return (type(t) not in (torch.Tensor, torch.nn.Parameter) or (t.requires_grad and torch.is_grad_enabled()) or
            torch.compiler.is_compiling() or torch.jit.is_tracing() or torch._C._len_torch_dispatch_stack() > 0 or
            torch._C._functorch.is_functorch_wrapped_tensor(t) or
            torch.autograd.forward_ad.unpack_dual(t).tangent is not None)


def _takes(scores, top):
    """Whether ``route_experts`` and its gradient take these scores."""
    return scores.shape[1] <= MOST_EXPERTS and top <= MOST_CHOSEN and _fits(scores)


def _sorted_choices(scores, top):
    """By torch: each token's weights and experts [T, top], the places of these choices in the rows' order, and the rows'
    ends."""
    p, chosen = torch.topk(scores.float(), top)
    p = torch.softmax(p, 1)
    expert, which = torch.sort(chosen.flatten(), stable=True)
    # (a count of each expert's rows would be a call that waits for the GPU)
    ends = torch.searchsorted(expert, torch.arange(scores.shape[1], device=expert.device), right=True, out_int32=True)
    return p, chosen, which, ends


def routing(scores, top):
    """``route_experts``, or the same from torch (without the loss; of equal scores any comes first): for more experts or
    choices than it takes, and where torch follows the scores, so that ``p`` carries their gradient."""
    return _routing(scores, top, _watched(scores))


def _routing(scores, top, followed):
    if not followed and _takes(scores, top):
        return route_experts(scores, top)
    p, chosen, which, ends = _sorted_choices(scores, top)
    row = torch.empty(which.shape[0], dtype=torch.int32, device=which.device)
    row[which] = torch.arange(which.shape[0], dtype=torch.int32, device=which.device)
    return Routing(chosen.int(), p, row.view(chosen.shape), (which // top).int(), torch.diff(ends, prepend=ends.new_zeros(1)),
                   ends, None)


def route(scores, top):
    """The rows of a grouped product for each token's ``top`` experts: ``token`` (the token of each row, rows sorted
    by expert), ``ends`` (int32, for the operators), ``p`` (its weight, with the gradient of scores that require one) and
    ``which`` (its place in [T, top])."""
    if _watched(scores) or not _takes(scores, top):
        p, _, which, ends = _sorted_choices(scores, top)
        return which // top, ends, p.flatten()[which], which
    r = route_experts(scores, top)
    row = r.row.flatten().long()
    which = torch.empty_like(row)
    which[row] = torch.arange(row.shape[0], device=row.device)
    return r.token.long(), r.ends, r.p.flatten()[which], which


def _balance(scores, counts, top):
    """What the balance loss is made of, by torch: its factor, each token's softmax over all experts (zeros where all its
    scores are -inf), and the experts' counts."""
    T, E = scores.shape
    v = scores.float()
    q = torch.where(v.amax(1, keepdim=True) == -torch.inf, 0.0, torch.softmax(v, 1))
    return E / (top * max(T, 1) ** 2), q, counts.float()


def balance_loss(scores, r):
    """The balance loss of the routing ``r`` of these scores, where ``routing`` left it out too."""
    if r.loss is not None:
        return r.loss
    factor, q, c = _balance(scores, r.counts, r.p.shape[1])
    return factor * (c * q.sum(0)).sum()


def routing_backward(dp, scores, r, dloss, dtype):
    """``route_experts_backward`` of the routing ``r``, or for more experts or choices than that takes the same from
    torch."""
    top = r.p.shape[1]
    if _takes(scores, top):
        return route_experts_backward(dp, scores, r.expert, r.p, r.counts, dloss, dtype=dtype)
    factor, q, c = _balance(scores, r.counts, top)
    ds = dloss * factor * q * (c - (q * c).sum(1, keepdim=True))
    return ds.scatter_add(1, r.expert.long(), r.p * (dp - (r.p * dp).sum(1, keepdim=True))).to(dtype)


def quantize_family(w):
    """Matrices [E, N, K] as float8_e4m3fn with a scale per 128 x 128 block, laid out once."""
    q, s = zip(*(quantize_fp8(m, block_rows=128) for m in w))
    return torch.stack([m.view(torch.uint8) for m in q]).view(torch.float8_e4m3fn), torch.stack(s)


def _normed(x, norm, bias, residual, quantize=False):
    if bias is None:
        return rmsnorm(x, norm, residual, quantize=quantize)
    return layernorm(x, norm, bias, residual, quantize=quantize)


class Served:
    """The block's weights in 8 bits: ``norm`` [D] (with ``bias`` [D] a layer norm's), ``router`` [E, D], ``w1``
    [E, D, F], ``w2`` [E, F, D]."""

    def __init__(self, norm, router, w1, w2, top=2, bias=None):
        self.norm, self.bias, self.top = norm, bias, top
        self.router = quantize_fp8(router, block_rows=128)
        self.w1 = quantize_family(w1.transpose(1, 2).contiguous())
        self.w2 = quantize_family(w2.transpose(1, 2).contiguous())

    def step(self, x, residual):
        """(out [T, D] float32, the sum that was normed): any number of tokens, one among them."""
        n = _normed(x, self.norm, self.bias, residual, quantize=True)
        r = _routing(matmul_fp8(n.out, n.scale, *self.router), self.top, False)
        rows = n.out.view(torch.uint8)[r.token].view(torch.float8_e4m3fn)
        h = matmul_grouped_fp8(rows, n.scale[r.token], *self.w1, r.ends, relu=True, dtype=torch.bfloat16)
        y = matmul_grouped_fp8(*quantize_fp8(h), *self.w2, r.ends, dtype=torch.bfloat16)
        return combine_experts(y, r.row, r.p), n.residual


#: What ``train_step`` returns where more than the experts is trained: its result, the gradients (None for what the block
#: does not have), and the balance loss.  ``dshared`` holds the gradients of (v1, c1, v2, c2).
TrainStep = namedtuple("TrainStep", "out dx dnorm dw1 dw2 dbias drouter dshared loss")


def train_step(x, residual, norm, router, w1, w2, dout, top=2, bias=None, balance=None, shared=None,
               activation="gelu_tanh"):
    """Forward and backward in bfloat16 for the output's gradient ``dout`` [T, D].

    Returns (out, gradients of x (the residual's is the same), norm, w1, w2), the routing taken as given; of a router
    that requires a gradient ``out`` carries it, through the weights of the chosen experts (by torch's products).  With
    ``bias`` [D] the norm is a layer norm; with the number ``balance`` the router is trained too, through the weights
    of the chosen experts and ``balance`` times the balance loss, its gradient a result like the others and ``out`` without
    one; ``shared`` = (v1 [D, S], c1 [S], v2 [S, D], c2 [D]) is an expert for every token.  With any of these the result is a
    ``TrainStep``."""
    bf16 = torch.bfloat16
    dout = dout if _fits(dout) else dout.float().contiguous()
    router = router if balance is None else router.detach()
    router = router if _fits(router) else router.contiguous()
    n = _normed(x, norm, bias, residual)
    followed = _watched(router)
    own = router.dtype == bf16 and not followed
    scores = linear(n.out, router, transpose_b=True) if own else n.out.float() @ router.float().t()
    r = _routing(scores, top, followed)
    rows = n.out[r.token]
    h = matmul_grouped(rows, w1, r.ends, relu=True, dtype=bf16)
    y = matmul_grouped(h, w2, r.ends, dtype=bf16)
    if followed:
        out = (y.float()[r.row.long()] * r.p[:, :, None]).sum(1)
        r = r._replace(p=r.p.detach())
    else:
        out = combine_experts(y, r.row, r.p)
    dense = dshared = drouter = None
    if shared is not None:
        v1, c1, v2, c2 = shared
        dense, z = linear(n.out, v1, c1, activation=activation, keep=True, dtype=bf16)
        out = out + linear(dense, v2, c2) if followed else linear(dense, v2, c2, residual=out)

    dy, dp = combine_experts_backward(dout, y, r.row, r.token, r.p)
    dw2 = matmul_grouped_wgrad(h, dy, r.ends)
    dh = matmul_grouped(dy, w2, r.ends, transpose_b=True, dtype=bf16)
    dh = torch.where(h > 0, dh, torch.zeros_like(dh))
    dw1 = matmul_grouped_wgrad(rows, dh, r.ends)
    dn = combine_experts(matmul_grouped(dh, w1, r.ends, transpose_b=True), r.row)
    if balance is not None:
        ds = routing_backward(dp, scores, r, float(balance), bf16 if own else torch.float32)
        if own:
            drouter = linear_wgrad(ds, n.out)
            dn = linear(ds, router, residual=dn)
        else:
            # (as its scores, no router is rounded to bf16, nor what reaches it)
            drouter = ds.t() @ n.out.float()
            dn = torch.addmm(dn, ds, router.float())
    if shared is not None:
        d2, dc2 = activation_backward(dout, None, None)
        d1, dc1 = activation_backward(linear(d2, v2, transpose_b=True, dtype=bf16), z, activation)
        dshared = (linear_wgrad(n.out, d1), dc1, linear_wgrad(dense, d2), dc2)
        dn = linear(d1, v1, transpose_b=True, residual=dn)
    dn = dn.to(x.dtype)
    if bias is None:
        dbias = None
        dx, dnorm = rmsnorm_backward(dn, n.residual, norm, n.rstd)
    else:
        dx, dnorm, dbias = layernorm_backward(dn, n.residual, norm, n.mean, n.rstd)
    if bias is None and balance is None and shared is None:
        return out, dx, dnorm, dw1, dw2
    return TrainStep(out, dx, dnorm, dw1, dw2, dbias, drouter, dshared, balance_loss(scores, r))


def weights(E, D, F, device="cuda", seed=0):
    g = torch.Generator(device=device).manual_seed(seed)

    def normal(*shape):
        return torch.randn(*shape, device=device, generator=g)

    return ((1 + 0.1 * normal(D)).bfloat16(), (normal(E, D) / D ** 0.5).bfloat16(),
            (normal(E, D, F) / D ** 0.5).bfloat16(), (normal(E, F, D) / F ** 0.5).bfloat16())


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--tokens", type=int, default=8192)
    ap.add_argument("--experts", type=int, default=16)
    ap.add_argument("--width", type=int, default=1024)
    ap.add_argument("--hidden", type=int, default=2048)
    ap.add_argument("--steps", type=int, default=20)
    a = ap.parse_args()
    norm, router, w1, w2 = weights(a.experts, a.width, a.hidden)
    served = Served(norm, router, w1, w2)

    def timed(what, f):
        for _ in range(3):
            f()
        torch.cuda.synchronize()
        t = time.perf_counter()
        for _ in range(a.steps):
            f()
        torch.cuda.synchronize()
        print("%-32s %.3f ms a step" % (what, (time.perf_counter() - t) / a.steps * 1e3), flush=True)

    for tokens in (1, a.tokens):
        x, r = (torch.randn(tokens, a.width, device="cuda").bfloat16() for _ in range(2))
        timed("serving %d token(s), 8 bits" % tokens, lambda: served.step(x, r))
    timed("training %d tokens, bfloat16" % a.tokens, lambda: train_step(x, r, norm, router, w1, w2, x))
    D, S = a.width, a.hidden
    shared = ((torch.randn(D, S, device="cuda") / D ** 0.5).bfloat16(), torch.zeros(S, device="cuda"),
              (torch.randn(S, D, device="cuda") / S ** 0.5).bfloat16(), torch.zeros(D, device="cuda"))
    timed("with its router and a shared expert",
          lambda: train_step(x, r, norm, router, w1, w2, x, bias=torch.zeros_like(norm), balance=0.01, shared=shared))


if __name__ == "__main__":
    main()

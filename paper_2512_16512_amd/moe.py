"""A mixture-of-experts block on the norm, 8-bit and grouped operators: one step
of serving in 8 bits and one of training in bfloat16, as a program would make
them.

    h = x + residual,  y = rmsnorm(h),  scores = y @ router.T
    out[t] = sum over t's top experts e of  p[t, e] * relu(y[t] @ w1[e]) @ w2[e]

``python -m paper_2512_16512_amd.moe`` runs both on random weights and prints
what a step takes.  Routing (top-k, sorting the rows by expert) and the weighted
sum over a token's experts are torch's.
"""
from __future__ import annotations

import argparse
import time

import torch

from . import (matmul_fp8, matmul_grouped, matmul_grouped_fp8, matmul_grouped_wgrad, quantize_fp8, rmsnorm,
               rmsnorm_backward)


def route(scores, top):
    """The rows of a grouped product for each token's ``top`` experts: ``token`` (the token of each row, rows sorted
    by expert), ``ends`` (int32, for the operators), ``p`` (its weight) and ``which`` (its place in [T, top])."""
    p, expert = torch.topk(scores.float(), top)
    p = torch.softmax(p, 1)
    expert, which = torch.sort(expert.flatten(), stable=True)
    # (a count of each expert's rows would be a call that waits for the GPU)
    ends = torch.searchsorted(expert, torch.arange(scores.shape[1], device=expert.device), right=True, out_int32=True)
    return which // top, ends, p.flatten()[which], which


def sum_experts(rows, which, T):
    """The sum of each token's rows, which go to the places ``which`` of [T, top]: in the order of its experts whatever
    the run (sums by atomics would give a token of three experts or more other bits from call to call)."""
    placed = torch.empty_like(rows)
    placed[which] = rows
    return placed.view(T, rows.shape[0] // max(T, 1), rows.shape[1]).sum(1)


def quantize_family(w):
    """Matrices [E, N, K] as float8_e4m3fn with a scale per 128 x 128 block, laid out once."""
    q, s = zip(*(quantize_fp8(m, block_rows=128) for m in w))
    return torch.stack([m.view(torch.uint8) for m in q]).view(torch.float8_e4m3fn), torch.stack(s)


class Served:
    """The block's weights in 8 bits: ``norm`` [D], ``router`` [E, D], ``w1`` [E, D, F], ``w2`` [E, F, D]."""

    def __init__(self, norm, router, w1, w2, top=2):
        self.norm, self.top = norm, top
        self.router = quantize_fp8(router, block_rows=128)
        self.w1 = quantize_family(w1.transpose(1, 2).contiguous())
        self.w2 = quantize_family(w2.transpose(1, 2).contiguous())

    def step(self, x, residual):
        """(out [T, D] float32, the sum that was normed): any number of tokens, one among them."""
        n = rmsnorm(x, self.norm, residual, quantize=True)
        token, ends, p, which = route(matmul_fp8(n.out, n.scale, *self.router), self.top)
        rows = n.out.view(torch.uint8)[token].view(torch.float8_e4m3fn)
        h = matmul_grouped_fp8(rows, n.scale[token], *self.w1, ends, relu=True, dtype=torch.bfloat16)
        y = matmul_grouped_fp8(*quantize_fp8(h), *self.w2, ends, dtype=torch.bfloat16)
        return sum_experts(y.float() * p[:, None], which, x.shape[0]), n.residual


def train_step(x, residual, norm, router, w1, w2, dout, top=2):
    """Forward and backward in bfloat16 for the output's gradient ``dout`` [T, D].  Returns (out, gradients of x (the
    residual's is the same), norm, w1, w2); the routing is taken as given."""
    n = rmsnorm(x, norm, residual)
    T = x.shape[0]
    token, ends, p, which = route(n.out.float() @ router.float().t(), top)
    rows = n.out[token]
    h = matmul_grouped(rows, w1, ends, relu=True, dtype=torch.bfloat16)
    y = matmul_grouped(h, w2, ends, dtype=torch.bfloat16)
    out = sum_experts(y.float() * p[:, None], which, T)

    dy = (dout.float()[token] * p[:, None]).bfloat16()
    dw2 = matmul_grouped_wgrad(h, dy, ends)
    dh = matmul_grouped(dy, w2, ends, transpose_b=True, dtype=torch.bfloat16)
    dh = torch.where(h > 0, dh, torch.zeros_like(dh))
    dw1 = matmul_grouped_wgrad(rows, dh, ends)
    drows = matmul_grouped(dh, w1, ends, transpose_b=True)
    dn = sum_experts(drows, which, T).to(x.dtype)
    dx, dnorm = rmsnorm_backward(dn, n.residual, norm, n.rstd)
    return out, dx, dnorm, dw1, dw2


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


if __name__ == "__main__":
    main()

"""Vocabulary entries that every token finds improbable have a gradient all the same."""
import math

import pytest
import torch

from paper_2312_06881_amd import nn
from tests.test_gpu_loss import DTYPES, BF

pytestmark = pytest.mark.gpu


def rare(M, n, V, dtype, first, seed=0):
    """Entries from ``first`` on have logits of 0 down to -80 and less, step by step; no target is among them."""
    g = torch.Generator().manual_seed(seed + M + n + V)
    x = torch.randn(M, n, generator=g)
    x[:, 0] = 8.0
    w = torch.randn(V, n, generator=g) / math.sqrt(n)
    w[:, 0] = 0.0
    w[first:, 0] = -torch.arange(V - first).remainder(81) / 8
    t = torch.randint(0, first, (M,), generator=g)
    t[3::7] = -100
    return x.to(dtype), w.to(dtype), t


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("M,n,V,first,reduction", [(1, 64, 300, 100, "sum"), (100, 72, 600, 300, "mean"), (300, 64, 1500, 40, "none"),
                                                   (2100, 64, 200000, 120000, "mean"), (5000, 128, 3000, 1000, "mean")])
def test_rows_keep_their_relative_precision(M, n, V, first, reduction, dtype):
    # A row's dw = sum_m G x is measured by its own terms.  G is off by its logit's error (6 sqrt(n) 2^-24 of the sum of the
    # products' magnitudes, and 2^-22 of what z log2(e) - lse log2(e) is formed from) and, with bf16 operands, as the
    # tokens are, by fp16's half step of 2^-11, of either sign.  fp16's smallest step is 2^-40 of the scale that a row's
    # largest G has at least 2^-24 of, so 2^-16 of that value.
    x, w, t = rare(M, n, V, dtype, first)
    a, b, td = x.cuda().requires_grad_(True), w.cuda().requires_grad_(True), t.cuda()
    loss = nn.linear_cross_entropy(a, b, td, reduction=reduction)
    dx, dw = torch.autograd.grad(loss, (a, b), torch.ones_like(loss))
    again = torch.autograd.grad(nn.linear_cross_entropy(a, b, td, reduction=reduction), (a, b), torch.ones_like(loss))
    assert torch.equal(dx, again[0]) and torch.equal(dw, again[1])
    used = (td >= 0).nonzero().view(-1)
    xd, wd = a.detach().double()[used], b.detach().double()
    z = xd @ wd.t()
    lse = torch.logsumexp(z, 1)
    dz = 6 * math.sqrt(n) * 2.0 ** -24 * (xd.abs() @ wd.abs().t()) + 2.0 ** -22 * (z.abs() + lse.abs()[:, None] + 1)
    p = torch.exp(z - lse[:, None])
    hot = torch.zeros_like(p)
    hot[torch.arange(len(used), device="cuda"), td[used]] = 1.0
    G = p - hot
    E = p * dz * 2 + 2.0 ** -23 * hot
    del z, dz, p, hot
    s = 1.0 / max(1, len(used)) if reduction == "mean" else 1.0
    want, terms = s * (G.t() @ xd), s * (G.t().abs() @ xd.abs())
    tol = s * (E.t() @ xd.abs()) + 6 * math.sqrt(max(1, len(used))) * 2.0 ** -24 * terms + 2.0 ** -24 * want.abs()
    # What is below fp32's (and bf16's) smallest normal number, 2^-126, may become zero: with bf16 operands a probability,
    # and the result; in fp32 each of the three parts of a G, and each of the six products with a token's parts.
    tol += s * 2.0 ** -125 * xd.abs().sum(0) + 2.0 ** -126 if dtype is BF else 2.0 ** -123 * (xd.abs() + 1).sum(0)
    if dtype is BF:
        top = G.abs().amax(0) if len(used) else torch.zeros(V, device="cuda", dtype=torch.float64)
        tol += 2.0 ** -8 * want.abs() + 6 * 2.0 ** -10 * s * ((G * G).t() @ (xd * xd)).sqrt()
        tol += s * 2.0 ** -16 * top[:, None] * xd.abs().sum(0) + s * 2.0 ** -39 * G.abs().sum(0)[:, None] * xd.abs().sum(0)
    off = (dw.double() - want).abs()
    assert (off <= tol).all(), float((off / tol).max())
    if len(used):
        assert dw[first:].any(1).float().mean() > 0.9


def test_captured_steps_with_rare_rows():
    from paper_2312_06881_amd import lm

    def step(s):
        loss, lse, count = lm.linear_cross_entropy(*s, keep=True)
        return [loss, *lm.linear_cross_entropy_backward(torch.ones_like(loss), *s, lse, count)]

    a, b = ([t.cuda() for t in rare(700, 64, 2000, BF, first, seed=first)] for first in (300, 1500))
    s = [t.clone() for t in a]
    step(s)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step(s)
    for new in (b, a, b, b):
        for t, u in zip(s, new):
            t.copy_(u)
        graph.replay()
        for x, y in zip(got, step(new)):
            assert torch.equal(x, y)


def test_rare_rows_without_the_tokens_gradient():
    x, w, t = rare(400, 72, 900, BF, 200)
    b = w.cuda().requires_grad_(True)
    dw, = torch.autograd.grad(nn.linear_cross_entropy(x.cuda(), b, t.cuda()), b)
    a = x.cuda().requires_grad_(True)
    both = torch.autograd.grad(nn.linear_cross_entropy(a, b, t.cuda()), (a, b))
    assert torch.equal(dw, both[1])
    dx, = torch.autograd.grad(nn.linear_cross_entropy(a, w.cuda(), t.cuda()), a)
    assert torch.equal(dx, both[0])

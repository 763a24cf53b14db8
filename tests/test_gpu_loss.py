"""linear_cross_entropy on the GPU against its definition in 64 bits.

fp32 sums of n products are taken to be within 6 sqrt(n) 2^-24 of the sum of the products' magnitudes
(rounding errors of either sign add up like a random walk; its own bound n 2^-24 is never nearly reached).
With bf16 operands the logits' gradient and the token (times the loss's gradient) are rounded to fp16 before they
are multiplied: each term of dX and dW is off by up to 2 2^-11 of itself, of either sign, together 6 2^-10 times
the root of the sum of their squares.  fp16's smallest step is 2^-24, so a value held as itself times 2^15, as G is, is
also off by up to 2^-40, and one of a column whose largest magnitude c was taken to 2^14 or more by up to c 2^-39.
"""
import math

import pytest
import torch

from paper_2312_06881_amd import nn

pytestmark = pytest.mark.gpu
BF, F = torch.bfloat16, torch.float32
DTYPES = [F, BF]


def make(M, n, V, dtype, seed=0, ignored=0.25, spread=2.0):
    g = torch.Generator().manual_seed(seed + 31 * M + 7 * n + V)
    w = (torch.randn(V, n, generator=g) * spread / math.sqrt(n)).to(dtype)
    t = torch.randint(0, V, (M,), generator=g)
    x = (torch.randn(M, n, generator=g) + w[t].float()).to(dtype)
    t = torch.where(torch.rand(M, generator=g) < ignored, torch.full_like(t, -100), t)
    return x, w, t


def check(x, w, t, reduction="mean", ignore=-100, dloss=None, no_grad=False):
    M, n = x.shape
    V = w.shape[0]
    xd, wd = x.cuda().double(), w.cuda().double()
    td = t.cuda()
    counts = (td >= 0) & (td < V) & (td != ignore)
    at = torch.where(counts, td, 0)
    z = xd @ wd.t()
    zmag = (xd.abs() @ wd.abs().t()).amax(1) if V else 0
    dz = 6 * math.sqrt(n) * 2.0 ** -24 * zmag + 2.0 ** -21       # of a logit; and of exp, log and the sum over tiles
    lse = torch.logsumexp(z, 1)
    each = torch.where(counts, lse - z.gather(1, at[:, None])[:, 0], 0.0)
    tol = torch.where(counts, 2 * dz + 2.0 ** -23 * (lse.abs() + each.abs()), 0.0)
    k = int(counts.sum())
    if reduction == "none":
        loss = each
    else:
        div = k if reduction == "mean" and k else 1
        loss, tol = each.sum() / div, tol.sum() / div + 2.0 ** -23 * each.sum().abs() / div
    a, b = x.cuda(), w.cuda()
    if no_grad:
        with torch.no_grad():
            got = nn.linear_cross_entropy(a, b, td, ignore, reduction)
        assert ((got.double() - loss).abs() <= tol).all()
        return got
    a.requires_grad_(True), b.requires_grad_(True)
    got = nn.linear_cross_entropy(a, b, td, ignore, reduction)
    assert got.dtype is F and got.shape == loss.shape
    assert ((got.double() - loss).abs() <= tol).all(), float(((got.double() - loss).abs() - tol).max())
    g = torch.ones_like(got) if dloss is None else dloss.cuda()
    dx, dw = torch.autograd.grad(got, (a, b), g)
    scale = g.double().expand(M) if reduction != "none" else g.double()
    scale = torch.where(counts, scale / (k if reduction == "mean" and k else 1), 0.0)
    p = torch.exp(z - lse[:, None])
    hot = torch.zeros_like(p).scatter_(1, at[:, None], 1.0)
    G = scale[:, None] * (p - hot)
    Gm = scale.abs()[:, None] * ((2 * dz[:, None] + 2.0 ** -22) * p + 2.0 ** -23 * (p + hot))  # how far G's values are off
    half = 2.0 ** -10 if x.dtype is BF else 0.0
    for name, out, A, B, E in (("dx", dx, G, wd, Gm), ("dw", dw, G.t().contiguous(), xd, Gm.t().contiguous())):
        want = A @ B
        assert out.dtype is x.dtype and out.shape == want.shape
        tol = (x.dtype is BF) * 2.0 ** -8 * want.abs() + 2.0 ** -24 * want.abs() + E @ B.abs()
        if x.dtype is BF:
            P = (p - hot).abs()
            Sx, Sc = scale.abs()[:, None] * xd.abs(), (scale.abs()[:, None] * xd.abs()).amax(0)
            if name == "dx":
                tol += scale.abs()[:, None] * (2.0 ** -40 * wd.abs().sum(0) + 2.0 ** -39 * P.sum(1)[:, None] * wd.abs().amax(0))
            else:
                tol += 2.0 ** -40 * Sx.sum(0) + 2.0 ** -39 * P.sum(0)[:, None] * Sc
        tol += 6 * half * ((A * A) @ (B * B)).sqrt() + 6 * math.sqrt(A.shape[1]) * 2.0 ** -24 * (A.abs() @ B.abs()) + 1e-37
        err = (out.double() - want).abs()
        assert (err <= tol).all(), (name, float((err / tol).max()))
    return got, dx, dw


SHAPES = [(1, 8, 2), (2, 64, 1), (5, 40, 77), (16, 64, 128), (33, 96, 300), (64, 1, 257), (127, 130, 1000), (130, 64, 513),
          (257, 128, 2049), (300, 1000, 777)]


@pytest.mark.parametrize("M,n,V", SHAPES)
@pytest.mark.parametrize("dtype", DTYPES)
def test_shapes(M, n, V, dtype):
    for reduction in ("mean", "sum", "none"):
        x, w, t = make(M, n, V, dtype)
        dloss = torch.randn(M, generator=torch.Generator().manual_seed(1)) if reduction == "none" else torch.tensor(1.7)
        check(x, w, t, reduction, dloss=dloss)
        check(x, w, t, reduction, no_grad=True)


@pytest.mark.parametrize("dtype", DTYPES)
def test_many_tiles(dtype):
    check(*make(1500, 192, 5003, dtype))
    check(*make(700, 320, 9000, dtype, spread=8.0))
    check(*make(4096, 64, 300, dtype))


@pytest.mark.parametrize("dtype", DTYPES)
def test_targets_that_do_not_count(dtype):
    x, w, t = make(90, 64, 500, dtype, ignored=0.0)
    t[::3] = 500
    t[1::9] = -1
    t[2] = 2 ** 62
    t[5] = -2 ** 62
    got, dx, dw = check(x, w, t)
    off = (t < 0) | (t >= 500)
    assert not dx[off.cuda()].any()
    each, _, _ = check(x, w, t, "none")
    assert not each[off.cuda()].any()
    # a token of the vocabulary may be the one to ignore
    t = torch.arange(90) % 7
    _, dx, _ = check(x, w, t, ignore=3)
    assert not dx[(t == 3).cuda()].any() and dx[(t == 4).cuda()].any()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("reduction", ["mean", "sum", "none"])
def test_none_counts(dtype, reduction):
    x, w, t = make(40, 64, 90, dtype, ignored=1.1)
    out = check(x, w, t, reduction)
    assert all(not v.any() for v in out)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("reduction", ["mean", "sum", "none"])
def test_empty_batch(dtype, reduction):
    w = torch.randn(37, 9, device="cuda", dtype=dtype, requires_grad=True)
    x = torch.empty(0, 9, device="cuda", dtype=dtype, requires_grad=True)
    loss = nn.linear_cross_entropy(x, w, torch.empty(0, dtype=torch.int64, device="cuda"), reduction=reduction)
    assert loss.shape == ((0,) if reduction == "none" else ()) and not loss.any()
    dx, dw = torch.autograd.grad(loss.sum(), (x, w))
    assert dx.shape == (0, 9) and not dw.any()


@pytest.mark.parametrize("dtype", DTYPES)
def test_large_logits(dtype):
    # one logit far above the others, or all far below zero: no overflow, no lost sum
    x, w, t = make(64, 64, 700, dtype, spread=300.0)
    check(x, w, t)
    w = -w.abs() - 4
    x = x.abs() + 1
    each = check(x, w, t, "none", no_grad=True)
    assert torch.isfinite(each).all()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("M", [70, 200, 600])
def test_nan_and_infinity_stay_in_their_tokens(dtype, M):
    x, w, t = make(M, 64, 400, dtype, ignored=0.0)
    t[11] = -100
    clean, dx0, _ = check(x, w, t, "none")
    x[3, 5] = float("nan")
    x[4, 6] = float("inf")
    x[11, 2] = float("nan")
    a, b = x.cuda().requires_grad_(True), w.cuda()
    each = nn.linear_cross_entropy(a, b, t.cuda(), reduction="none")
    dx, = torch.autograd.grad(each, a, torch.ones_like(each))
    ok = torch.ones(M, dtype=torch.bool, device="cuda")
    ok[[3, 4]] = False
    assert torch.equal(each[ok], clean[ok]) and torch.isnan(each[~ok]).all()
    assert torch.equal(dx[ok], dx0[ok]) and torch.isnan(dx[3]).all()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("ignored", [0.0, 0.02, 0.5, 0.97, 1.1])
def test_few_or_many_count(dtype, ignored):
    # enough tokens that those that count are gathered; a batch that begins and ends with others
    x, w, t = make(801, 72, 1100, dtype, ignored=ignored)
    if ignored > 0.1:
        t[:300] = -100
        t[790:] = -100
    check(x, w, t)
    check(x, w, t, "none", no_grad=True)


@pytest.mark.parametrize("M,n,V,dtype", [(4096, 64, 70001, BF), (1500, 72, 66000, F), (128, 8, 530000, F)])
def test_several_pieces_of_the_vocabulary(M, n, V, dtype):
    check(*make(M, n, V, dtype, ignored=0.1))


def test_many_splits_of_the_vocabulary():
    check(*make(260, 64, 40000, BF))
    check(*make(40, 192, 30000, BF))


@pytest.mark.parametrize("dtype", DTYPES)
def test_leading_dimensions_and_one_gradient_only(dtype):
    x, w, t = make(60, 64, 300, dtype)
    got, dx, dw = check(x, w, t)
    a = x.cuda().view(3, 20, 64)
    for leaf in ("x", "w"):
        p, q = a.clone().requires_grad_(leaf == "x"), w.cuda().requires_grad_(leaf == "w")
        loss = nn.linear_cross_entropy(p, q, t.cuda().view(3, 20))
        g, = torch.autograd.grad(loss, p if leaf == "x" else q)
        assert torch.equal(loss, got) and torch.equal(g.view(-1, 64), dx if leaf == "x" else dw)
    with torch.no_grad():
        each = nn.linear_cross_entropy(a, w.cuda(), t.cuda().view(3, 20), reduction="none")
    assert each.shape == (3, 20)


def test_module_with_a_shared_weight():
    e = torch.nn.Embedding(50, 64, device="cuda", dtype=DTYPES[-1])
    m = nn.LinearCrossEntropy(64, 50, weight=e.weight)
    t = torch.randint(0, 50, (4, 9), device="cuda")
    loss = m(e(t), t.roll(-1, 1))
    loss.backward()
    assert e.weight.grad.shape == (50, 64) and torch.isfinite(e.weight.grad.float()).all()
    assert len(list(m.parameters())) == 1

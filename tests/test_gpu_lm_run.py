"""Dropout, add_norm and the loss as they run together: a small language model of Dyad blocks against 64 bits, captured
steps, other streams, gradients of slices."""
import math

import pytest
import torch
import torch.utils.checkpoint

from paper_2312_06881_amd import lm, nn
from tests import lm_reference as ref

pytestmark = pytest.mark.gpu
BF, F = torch.bfloat16, torch.float32
D, FFN, DYAD, VOCAB, LAYERS, P = 64, 160, 4, 211, 3, 0.2


class Model(torch.nn.Module):
    """Embedding, LAYERS pre-norm blocks of DyadFF with dropout and sandwich norms, and the loss with the embedding's
    weight."""

    def __init__(self, dtype, variant="IT"):
        super().__init__()
        torch.manual_seed(1)
        kw = dict(device="cuda", dtype=dtype)
        self.embed = torch.nn.Embedding(VOCAB, D, **kw)
        with torch.no_grad():
            self.embed.weight.normal_(std=0.5)
        self.drop = nn.Dropout(P, seed=100)
        self.first = nn.AddNorm(D, **kw)
        self.joins = torch.nn.ModuleList(nn.AddNorm(D, post_norm="rms", gate=True, gate_init=0.75, p=P, seed=200 + i, **kw)
                                         for i in range(LAYERS))
        self.ffs = torch.nn.ModuleList(nn.DyadFF(D, FFN, DYAD, variant, **kw) for _ in range(LAYERS))
        self.loss = nn.LinearCrossEntropy(D, VOCAB, weight=self.embed.weight)

    def forward(self, tokens, targets):
        x, a = self.first(self.drop(self.embed(tokens)))
        for ff, join in zip(self.ffs, self.joins):
            x, a = join(x, ff(a))
        return self.loss(a, targets)


def dense(w1, w2, variant):
    """The weight [n_out, n_in] that a Dyad layer's components make up."""
    n, bo, bi = w1.shape
    i, j, k = torch.meshgrid(torch.arange(n), torch.arange(bo), torch.arange(bi), indexing="ij")
    one = (i * bo + j) * (n * bi) + i * bi + k
    row = j * n + i if variant in ("OT", "DT") else i * bo + j
    col = k * n + i if variant in ("IT", "DT") else i * bi + k
    W = torch.zeros(n * bo * n * bi, dtype=w1.dtype)
    W = W.index_add(0, one.flatten(), w1.flatten()).index_add(0, (row * (n * bi) + col).flatten(), w2.flatten())
    return W.view(n * bo, n * bi)


def exact(model, tokens, targets, variant):
    """The loss and its gradients in 64 bits through autograd, by parameter name."""
    p = {n: v.detach().cpu().double().requires_grad_(True) for n, v in model.named_parameters()}
    M = tokens.numel()

    def drop(x, layer):
        kept, scale = ref.keep_mask(M, D, P, layer.seed, layer.offset)
        return torch.where(kept, x * scale, 0.0)

    def norm(x, kind, w, b=None):
        if kind == "layer":
            x = x - x.mean(1, keepdim=True)
        x = x * (x.square().mean(1, keepdim=True) + 1e-5).rsqrt() * w
        return x if b is None else x + b

    x = drop(p["embed.weight"][tokens.cpu().view(-1)], model.drop)
    a = norm(x, "layer", p["first.weight"], p["first.bias"])
    for i in range(LAYERS):
        fc = [(dense(p[f"ffs.{i}.{n}.w1"], p[f"ffs.{i}.{n}.w2"], variant), p[f"ffs.{i}.{n}.bias"]) for n in ("fc1", "fc2")]
        h = a @ fc[0][0].t() + fc[0][1]
        y = (h * 0.5 * torch.erfc(-h / math.sqrt(2.0))) @ fc[1][0].t() + fc[1][1]
        z = drop(norm(y, "rms", p[f"joins.{i}.post_weight"]), model.joins[i].dropout)
        x = x + p[f"joins.{i}.gate"] * z
        a = norm(x, "layer", p[f"joins.{i}.weight"], p[f"joins.{i}.bias"])
    t = targets.cpu().view(-1)
    loss = torch.nn.functional.cross_entropy(a @ p["embed.weight"].t(), t)
    loss.backward()
    return loss.detach(), {n: v.grad for n, v in p.items()}


@pytest.mark.parametrize("variant", ["IT", "OT", "DT"])
@pytest.mark.parametrize("dtype,tol", [(F, 1e-4), (BF, 5e-2)])
def test_language_model(variant, dtype, tol):
    # tol: of each gradient's norm.  bf16 rounds every activation and gradient of 12 layers once, 2^-9 of itself at a
    # time and of either sign; 24 of them in a row add up to sqrt(24) 2^-9 = 1 %, and the last norms of a block of
    # rounded values scale that by up to 4.  fp32: 2^-24 in place of 2^-9, sums of hundreds of products.
    torch.manual_seed(2)
    tokens = torch.randint(0, VOCAB, (3, 23), device="cuda")
    targets = tokens.roll(-1, 1)
    targets[:, -1] = -100
    m = Model(dtype, variant)
    torch.manual_seed(5)
    loss = m(tokens, targets)
    loss.backward()
    want, grads = exact(m, tokens, targets, variant)
    assert abs(float(loss) - float(want)) <= tol * float(want)
    for n, v in m.named_parameters():
        g = v.grad.cpu().double()
        assert (g - grads[n]).norm() <= tol * grads[n].norm(), n
    # the same seed draws the same masks, another pass others, evaluation none
    torch.manual_seed(5)
    assert float(m(tokens, targets)) == float(loss)
    again = m(tokens, targets)
    assert float(again) != float(loss)
    m.eval()
    with torch.no_grad():
        assert float(m(tokens, targets)) == float(m(tokens, targets))


def test_checkpointed_layers_draw_the_same_masks():
    torch.manual_seed(3)
    join, drop = nn.AddNorm(48, p=0.4, device="cuda", dtype=F), nn.Dropout(0.3)
    x = torch.randn(30, 48, device="cuda", requires_grad=True)
    y = torch.randn(30, 48, device="cuda", requires_grad=True)

    def layer(x, y):
        h, out = join(x, drop(y))
        return h * out

    results = []
    for again in (False, True):
        torch.manual_seed(4)
        z = torch.utils.checkpoint.checkpoint(layer, x, y, use_reentrant=False) if again else layer(x, y)
        results.append([z.detach(), *torch.autograd.grad(z, (x, y, join.weight, join.bias), torch.ones_like(z))])
    for a, b in zip(*results):
        assert torch.equal(a, b)


def step_tensors(seed, dtype=BF, M=600, n=128, V=700):
    g = torch.Generator(device="cuda").manual_seed(seed)

    def t(*s):
        return torch.randn(*s, generator=g, device="cuda").to(dtype)

    return {"x": t(M, n), "y": t(M, n), "w": t(n), "b": t(n), "gate": t(4, n), "vocab": t(V, n) * 0.1,
            "t": torch.randint(-1, V, (M,), generator=g, device="cuda"), "dh": t(M, n)}


def whole_step(s, offset):
    """Forward and backward passes without autograd; every result."""
    kw = dict(post_norm="rms", post_weight=s["w"], gate=s["gate"], p=0.3, seed=5, offset=offset)
    h, out, stats, post_stats = lm.add_norm(s["x"], s["y"], "layer", s["w"], s["b"], keep=True, **kw)
    loss, lse, count = lm.linear_cross_entropy(out, s["vocab"], s["t"], keep=True)
    dout, dv = lm.linear_cross_entropy_backward(torch.ones_like(loss), out, s["vocab"], s["t"], lse, count)
    g = lm.add_norm_backward(s["dh"], dout, stats, post_stats, s["x"], s["y"], "layer", s["w"], s["b"], **kw)
    return [h, out, loss, dv, *g.values()]


@pytest.mark.parametrize("dtype", [F, BF])
def test_captured_step(dtype):
    s = step_tensors(1, dtype)
    offset = torch.zeros(1, dtype=torch.int64, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        whole_step(s, offset)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            got = whole_step(s, offset)
    other = step_tensors(9, dtype)
    for k in range(4):
        new = step_tensors(10 + k, dtype)
        for name in s:
            s[name].copy_(new[name])
        offset.fill_(k)
        torch.cuda.synchronize()
        graph.replay()
        whole_step(other, 3)                        # eager work beside it, on another stream
        torch.cuda.synchronize()
        for a, b in zip(got, whole_step(s, k)):
            assert torch.equal(a, b)


def test_two_captured_graphs_and_other_streams():
    a, b = step_tensors(1), step_tensors(2)
    want = [whole_step(a, 0), whole_step(b, 1)]
    torch.cuda.synchronize()
    graphs, got = [], []
    for s, k in ((a, 0), (b, 1)):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            got.append(whole_step(s, k))
        graphs.append(g)
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    for _ in range(3):
        for g, st in zip(graphs, streams):
            with torch.cuda.stream(st):
                g.replay()
        with torch.cuda.stream(streams[0]):
            eager = whole_step(b, 1)
        torch.cuda.synchronize()
        for x, y in zip(got + [eager], want + [want[1]]):
            assert all(torch.equal(p, q) for p, q in zip(x, y))


def test_gradients_of_slices_and_stacked_losses():
    # what autograd hands on is not always where the library takes it
    s = step_tensors(3, BF, 40, 33, 90)
    w = s["vocab"].requires_grad_(True)
    x = s["x"].requires_grad_(True)
    t = s["t"].abs()
    both = torch.stack([nn.linear_cross_entropy(x[:20], w, t[:20]), nn.linear_cross_entropy(x[21:], w, t[21:])])
    dx, dw = torch.autograd.grad((both * torch.tensor([1.0, 3.0], device="cuda")).sum(), (x, w))
    parts = []
    for sl, k in ((slice(0, 20), 1.0), (slice(21, 40), 3.0)):
        p, q = x.detach()[sl].clone().requires_grad_(True), w.detach().clone().requires_grad_(True)
        parts.append(torch.autograd.grad(nn.linear_cross_entropy(p, q, t[sl]) * k, (p, q)))
    assert torch.equal(dx[:20], parts[0][0]) and torch.equal(dx[21:], parts[1][0]) and not dx[20].any()
    assert torch.equal(dw, parts[0][1] + parts[1][1])
    # a norm of odd rows of a wider tensor, and a gradient that is a slice
    full = torch.cat([nn.add_norm(x[1:9], None, "rms")[1], nn.dropout(x[9:12], 0.5, 3)])
    g = torch.randn(11, 33, device="cuda").bfloat16()
    dx, = torch.autograd.grad(full, x, g)
    p = x.detach()[1:9].clone().requires_grad_(True)
    want, = torch.autograd.grad(nn.add_norm(p, None, "rms")[1], p, g[:8].clone())
    assert torch.equal(dx[1:9], want) and torch.equal(dx[9:12], lm.dropout(g[8:].clone(), 0.5, 3))


def test_double_backward_is_refused():
    s = step_tensors(4, F, 12, 16, 20)
    x = s["x"].requires_grad_(True)
    for out in (nn.add_norm(x, s["y"], "layer")[1].square().sum(),
                nn.linear_cross_entropy(x, s["vocab"], s["t"]).square()):
        g, = torch.autograd.grad(out, x, create_graph=True)
        with pytest.raises(RuntimeError):
            g.sum().backward()


def test_long_batches():
    # more tokens and values than 32 bits count in bytes: 300000 rows of 8192 in bf16
    M, n = 300000, 8192
    x = torch.ones((M, n), device="cuda", dtype=BF)
    x[-1] = 2.0
    x[-1, ::2] = 4.0
    h, out = nn.add_norm(x, x, "layer", None, None)
    assert torch.equal(h[-1], 2 * x[-1]) and torch.equal(h[7], 2 * x[7])
    assert torch.equal(out[-1, :4].float().cpu(), torch.tensor([1.0, -1.0, 1.0, -1.0])) and not out[M - 2].any()
    y = lm.dropout(x, 0.5, 11)
    kept, _ = ref.keep_mask(1, 8, 0.5, 11, 0)
    assert torch.equal((y[0, :8] != 0).cpu(), kept[0])
    words = ref.philox_words([((M - 1) * (n // 8)) & 0xffffffff, ((M - 1) * (n // 8)) >> 32, 0, 0], [11, 0])
    last = torch.tensor([((words[j // 2] >> (16 * (j % 2))) & 0xffff) >= 32768 for j in range(8)])
    assert torch.equal((y[-1, :8] != 0).cpu(), last)

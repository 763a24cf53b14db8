"""Dropout, add_norm and the loss without a GPU: the reference against autograd and published vectors, and refusals."""
import pytest
import torch

import paper_2312_06881_amd as dy
from paper_2312_06881_amd import lm, nn
from tests import lm_reference as ref

FAKE = 1 << 20     # a 16-byte-aligned non-NULL address; never dereferenced by rejected calls


def test_generator_known_answers():
    # the authors' published vectors of Philox-4x32-10
    assert ref.philox_words([0] * 4, [0] * 2) == [0x6627e8d5, 0xe169c58d, 0xbc57ac4c, 0x9b00dbd8]
    ones = 0xffffffff
    assert ref.philox_words([ones] * 4, [ones] * 2) == [0x408f276d, 0x41c83b0e, 0xa20bc7c6, 0x6d5451fd]


def test_mask_is_the_generators():
    seed, offset = 0x1234567890abcdef, 0xfedcba0987654321
    kept, scale = ref.keep_mask(3, 11, 0.25, seed, offset)
    assert scale == 65536 / (65536 - 16384)
    for row in range(3):
        for col in range(11):
            o = row * 2 + col // 8
            w = ref.philox_words([o, 0, offset & 0xffffffff, offset >> 32], [seed & 0xffffffff, seed >> 32])
            j = col % 8
            assert bool(kept[row, col]) == ((w[j // 2] >> (16 * (j % 2))) & 0xffff >= 16384)


@pytest.mark.parametrize("norm", ["layer", "rms"])
@pytest.mark.parametrize("post", ["layer", "rms", None])
@pytest.mark.parametrize("groups", [0, 1, 3])
def test_reference_gradients_are_autograds(norm, post, groups):
    g = torch.Generator().manual_seed(3)
    n, M = 21, 12

    def t(*s):
        return torch.randn(*s, generator=g, dtype=torch.float64)

    a = {"x": t(M, n), "y": t(M, n), "weight": t(n), "bias": t(n), "post_weight": t(n) if post else None,
         "post_bias": t(n) if post else None, "gate": None if not groups else t(n) if groups == 1 else t(groups, n)}
    dh, dout = t(M, n), t(M, n)
    kw = dict(xs=0.7, ys=-1.3, eps=1e-5, p=0.3, seed=5, offset=1)

    def call(v, **grads):
        return ref.add_norm(v["x"], v["y"], norm, v["weight"], v["bias"], post, v["post_weight"], v["post_bias"], v["gate"],
                            kw["xs"], kw["ys"], kw["eps"], kw["p"], kw["seed"], kw["offset"], **grads)

    leaves = {k: v.clone().requires_grad_(True) for k, v in a.items() if v is not None}
    r = call({k: leaves.get(k) for k in a})
    want = torch.autograd.grad((r["h"][0], r["out"][0]), list(leaves.values()), (dh, dout))
    got = call(a, dh=dh, dout=dout)
    for k, w in zip(leaves, want):
        assert torch.allclose(got[k][0], w, rtol=1e-11, atol=1e-11), k


def norm_args(**kw):
    v = dict(M=4, n=64, groups=1, stream_dtype=dy.BF16, dtype=dy.BF16, param_dtype=dy.BF16, norm=dy.NORM_LAYER,
             post=dy.NORM_RMS, x_scale=1.0, y_scale=1.0, eps=1e-5, p=0.1, seed=0, offset=0, offset_dev=None, x=FAKE, y=FAKE,
             weight=FAKE, bias=FAKE, post_weight=FAKE, post_bias=FAKE, gate=FAKE, h=FAKE, out=FAKE, stats=FAKE,
             post_stats=FAKE)
    v.update(kw)
    return dy.AddNormArgs(**v)


def grad_args(**kw):
    v = dict(dh=FAKE, dout=FAKE, dx=FAKE, dy=FAKE, dweight=FAKE, dbias=FAKE, dpost_weight=FAKE, dpost_bias=FAKE, dgate=FAKE)
    v.update(kw)
    return dy.AddNormGrads(**v)


BAD_BOTH = [(dict(M=-1), -1), (dict(n=0), -1), (dict(n=-8), -1), (dict(n=7), -2), (dict(n=16385), -2), (dict(groups=0), -1),
            (dict(groups=3), -1), (dict(M=2 ** 31), -1), (dict(stream_dtype=7), -4), (dict(dtype=-1), -4),
            (dict(param_dtype=2), -4), (dict(dtype=dy.F32), -4),
            (dict(stream_dtype=dy.F32, dtype=dy.F32, param_dtype=dy.BF16), -4), (dict(norm=3), -1), (dict(post=-1), -1),
            (dict(eps=-1.0), -1), (dict(eps=float("nan")), -1), (dict(p=-0.1), -1), (dict(p=1.5), -1),
            (dict(p=float("nan")), -1), (dict(weight=FAKE + 8), -3), (dict(offset_dev=FAKE + 4), -3)]


@pytest.mark.parametrize("kw,code", BAD_BOTH + [(dict(x=None), -1), (dict(out=None), -1), (dict(x=FAKE + 2), -3),
                                                (dict(norm=0, h=None), -1)])
def test_add_norm_forward_refuses(kw, code):
    assert dy.dyad_add_norm_forward(norm_args(**kw), None) == code


@pytest.mark.parametrize("kw,gkw,code", [(a, {}, c) for a, c in BAD_BOTH] + [
    (dict(h=None, x=None), {}, -1), (dict(stats=None), {}, -1), (dict(post_stats=None), {}, -1), (dict(norm=0), {}, -1),
    (dict(norm=0), dict(dout=None, dbias=None), -1), (dict(post=0), {}, -1), (dict(y=None), {}, -1),
    (dict(gate=None), {}, -1), ({}, dict(dx=FAKE + 4), -3), ({}, {}, -5)])
def test_add_norm_backward_refuses(kw, gkw, code):
    a, g = norm_args(**kw), grad_args(**gkw)
    if code != -5:
        size = 1 << 40
        assert dy.dyad_add_norm_backward(a, g, FAKE, size, None) == code
    else:
        need = dy.dyad_add_norm_workspace_bytes(a, g)
        assert need > 0
        assert dy.dyad_add_norm_backward(a, g, FAKE, need - 1, None) == -5
        assert dy.dyad_add_norm_backward(a, g, None, need, None) == -5
        assert dy.dyad_add_norm_backward(a, g, FAKE + 8, need, None) == -3


def test_null_structures():
    assert dy.dyad_add_norm_forward(None, None) == -1
    assert dy.dyad_add_norm_backward(norm_args(), None, FAKE, 1 << 30, None) == -1
    assert dy.dyad_add_norm_backward(None, grad_args(), FAKE, 1 << 30, None) == -1
    assert dy.dyad_add_norm_workspace_bytes(None, grad_args()) == 0
    assert dy.dyad_add_norm_workspace_bytes(norm_args(n=3), grad_args()) == 0


def test_add_norm_workspace():
    none = dict.fromkeys(("dweight", "dbias", "dpost_weight", "dpost_bias", "dgate"))
    assert dy.dyad_add_norm_workspace_bytes(norm_args(M=5000), grad_args(**none)) == 0
    some = dy.dyad_add_norm_workspace_bytes(norm_args(M=5000), grad_args())
    assert dy.dyad_add_norm_workspace_bytes(norm_args(M=5000, groups=5000), grad_args()) >= some
    assert some % 4 == 0 and some < 5 * 4 * 64 * 5000


@pytest.mark.parametrize("kw,code", [
    (dict(dtype=5), -4), (dict(rows=-1), -1), (dict(cols=0), -1), (dict(p=-0.5), -1), (dict(p=float("nan")), -1),
    (dict(p=1.01), -1), (dict(x=None), -1), (dict(y=None), -1), (dict(x=FAKE + 2), -3), (dict(off=FAKE + 4), -3),
    (dict(rows=2 ** 31), -1), (dict(cols=2 ** 31 - 8, rows=1), -1), (dict(rows=2 ** 30, cols=2 ** 12), -1), (dict(rows=0, x=None, y=None), 0)])
def test_dropout_refuses(kw, code):
    v = dict(rows=4, cols=8, dtype=dy.BF16, x=FAKE, p=0.5, off=None, y=FAKE)
    v.update(kw)
    assert dy.dyad_dropout(v["rows"], v["cols"], v["dtype"], v["x"], v["p"], 1, 2, v["off"], v["y"], None) == code


CE = dict(M=4, n=8, V=100, dtype=dy.F32, X=FAKE, W=FAKE, t=FAKE, red=dy.REDUCE_MEAN, loss=FAKE, lse=FAKE, count=FAKE, dX=FAKE,
          dW=FAKE, ws=FAKE, size=1 << 40)


@pytest.mark.parametrize("kw,code", [
    (dict(dtype=3), -4), (dict(M=-1), -1), (dict(n=0), -1), (dict(V=0), -1), (dict(M=2 ** 22 + 1), -2),
    (dict(V=2 ** 22 + 1), -2), (dict(M=2 ** 20, V=2 ** 18 + 1), -2), (dict(n=2 ** 20 + 1), -2), (dict(red=3), -1), (dict(X=None), -1), (dict(W=None), -1),
    (dict(t=None), -1), (dict(lse=None), -1), (dict(loss=None), -1), (dict(count=None), -1), (dict(X=FAKE + 8), -3),
    (dict(t=FAKE + 8), -3), (dict(ws=None), -5), (dict(size=8), -5), (dict(ws=FAKE + 4), -3)])
def test_linear_ce_refuses(kw, code):
    v = {**CE, **kw}
    assert dy.dyad_linear_ce_forward(v["M"], v["n"], v["V"], v["dtype"], v["X"], v["W"], v["t"], -100, v["red"], v["loss"],
                                     v["lse"], v["count"], v["ws"], v["size"], None) == code
    assert dy.dyad_linear_ce_backward(v["M"], v["n"], v["V"], v["dtype"], v["X"], v["W"], v["t"], -100, v["red"], v["lse"],
                                      v["count"], v["loss"], v["dX"], v["dW"], v["ws"], v["size"], None) == code
    if code != -5 and "lse" not in kw:
        size = dy.dyad_linear_ce_workspace_bytes(dy.CE_BACKWARD, v["M"], v["n"], v["V"], v["dtype"])
        assert (size == 0) == (v["dtype"] == 3 or v["M"] < 0 or v["n"] <= 0 or v["V"] <= 0 or code == -2)


def test_linear_ce_backward_of_nothing():
    assert dy.dyad_linear_ce_backward(4, 8, 100, dy.F32, FAKE, FAKE, FAKE, -100, dy.REDUCE_MEAN, FAKE, FAKE, FAKE, None, None,
                                      None, 0, None) == 0
    assert dy.dyad_linear_ce_workspace_bytes(2, 4, 8, 100, dy.F32) == 0


def test_helpers_refuse():
    x, w, t = torch.zeros(4, 16), torch.zeros(50, 16), torch.zeros(4, dtype=torch.int64)
    for p in (-0.1, 1.1, float("nan")):
        with pytest.raises(ValueError):
            nn.dropout(x, p, 1)
    for kw in (dict(seed=-1), dict(seed=2 ** 64), dict(seed=1, offset=-1), dict(seed=1, offset=torch.zeros(2, dtype=torch.int64)),
               dict(seed=1, offset=torch.zeros(1))):
        with pytest.raises(ValueError):
            nn.dropout(x, 0.5, **kw)
    with pytest.raises(TypeError):
        nn.dropout(x.half(), 0.5, 1)
    with pytest.raises(ValueError, match="device tensors"):
        nn.dropout(x, 0.5, 1)
    for args, kw in (((x, x[:2]), {}), ((x, x, "group"), {}), ((x, x), dict(post_norm="l2")), ((x,), dict(gate=x[0])),
                     ((x,), dict(p=0.5)), ((x,), dict(post_norm="rms")), ((x, x, None, x[0]), {}),
                     ((x, x, "layer", x[0, :8]), {}), ((x, x), dict(post_weight=x[0])), ((x, x), dict(gate=x[0, :8])),
                     ((x, x), dict(gate=x[:3])), ((x, x), dict(gate=x[:0])), ((x, x), dict(dtype=torch.bfloat16))):
        with pytest.raises(ValueError):
            lm.add_norm(*args, **kw)
    with pytest.raises(TypeError):
        lm.add_norm(x, x, "layer", x[0], x[0].bfloat16())
    for args in ((x, w[:, :8], t), (x, w, t[:3]), (x, w, t.int()), (x[0], w, t)):
        with pytest.raises(ValueError):
            lm.linear_cross_entropy(*args)
    with pytest.raises(ValueError):
        nn.linear_cross_entropy(x, w, t, reduction="max")
    with pytest.raises(ValueError):
        nn.linear_cross_entropy(x, w, t.view(2, 2))
    with pytest.raises(TypeError):
        lm.linear_cross_entropy(x, w.bfloat16(), t)
    with pytest.raises(ValueError, match="device tensors"):
        nn.linear_cross_entropy(x, w, t)
    with pytest.raises(ValueError):
        nn.Dropout(2.0)
    with pytest.raises(ValueError):
        nn.AddNorm(8, norm="batch")
    with pytest.raises(ValueError):
        nn.LinearCrossEntropy(16, 50, weight=torch.nn.Parameter(torch.zeros(49, 16)))


def test_modules_on_the_cpu():
    d = nn.Dropout(0.1, seed=5)
    torch.manual_seed(3)
    first = [d.next_offset() for _ in range(3)]
    torch.manual_seed(3)
    assert first == [d.next_offset() for _ in range(3)] and len(set(first)) == 3 and d.offset == first[-1]
    x = torch.ones(3)
    assert d.eval()(x) is x
    c = nn.Dropout(0.1, capturable=True)
    assert "calls" in c.state_dict() and int(c.next_offset()) == 0 and int(c.next_offset()) == 1
    m = nn.AddNorm(8, post_norm="layer", gate=True)
    assert sorted(n for n, _ in m.named_parameters()) == ["bias", "gate", "post_bias", "post_weight", "weight"]
    m = nn.AddNorm(8, norm="rms", bias=False)
    assert [n for n, _ in m.named_parameters()] == ["weight"]

"""add_norm on the GPU against its definition in 64 bits (lm_reference)."""
import itertools

import pytest
import torch

from tests import lm_reference as ref
from paper_2312_06881_amd import lm, nn

pytestmark = pytest.mark.gpu

BF, F = torch.bfloat16, torch.float32
TYPES = {"bf16": (BF, BF, BF), "bf16_f32params": (BF, BF, F), "f32_stream": (F, BF, BF), "f32_stream_params": (F, BF, F),
         "f32": (F, F, F)}


def make(M, n, types, norm="layer", post=None, gate=0, bias=True, seed=0, with_y=True, shift=0.0):
    st, bt, pt = TYPES[types]
    g = torch.Generator().manual_seed(1000 * seed + M + n)

    def t(shape, std, mean, dt):
        return (torch.randn(shape, generator=g) * std + mean).to(dt)

    d = {"x": t((M, n), 2.0, shift, st), "y": t((M, n), 1.0, 0.25, bt) if with_y else None, "norm": norm, "post_norm": post,
         "weight": t((n,), 0.3, 1.0, pt) if norm else None, "bias": t((n,), 0.3, 0.0, pt) if norm and bias else None,
         "post_weight": t((n,), 0.3, 1.0, pt) if post else None, "post_bias": t((n,), 0.3, 0.0, pt) if post and bias else None,
         "gate": None}
    if gate:
        d["gate"] = t((n,) if gate == 1 else (gate, n), 0.5, 0.5, pt)
    return d, t((M, n), 1.0, 0.0, st), t((M, n), 1.0, 0.0, bt)


NAMES = ("x", "y", "weight", "bias", "post_weight", "post_bias", "gate")


def reference(d, kw, dh, dout, kept_h=None):
    v = {k: None if d[k] is None else d[k].double() for k in NAMES}
    full = dict(x_scale=1.0, y_scale=1.0, eps=1e-5, p=0.0, seed=0, offset=0)
    full.update(kw)
    return ref.add_norm(v["x"], v["y"], d["norm"], v["weight"], v["bias"], d["post_norm"], v["post_weight"], v["post_bias"],
                        v["gate"], full["x_scale"], full["y_scale"], full["eps"], full["p"], full["seed"], full["offset"],
                        kept_h, None if dh is None else dh.double(), None if dout is None else dout.double())


def step(d, kw, dh, dout):
    """h, out and the gradients through autograd, by name."""
    leaves = {k: d[k].cuda().requires_grad_(True) for k in NAMES if d[k] is not None}
    a = {k: leaves.get(k) for k in NAMES}
    h, out = nn.add_norm(a["x"], a["y"], d["norm"], a["weight"], a["bias"], post_norm=d["post_norm"],
                         post_weight=a["post_weight"], post_bias=a["post_bias"], gate=a["gate"], **kw)
    pairs = [(o, g.cuda()) for o, g in ((h, dh), (out, dout)) if o is not None and g is not None]
    grads = torch.autograd.grad([o for o, _ in pairs], list(leaves.values()), [g for _, g in pairs], allow_unused=True)
    return {"h": h, "out": out, **dict(zip(leaves, grads))}


def compare(d, kw, dh, dout, what=""):
    got = step(d, kw, dh, dout)
    # an fp32 stream's h is read again by the backward pass, a bf16 one's formed again
    want = reference(d, kw, dh, dout, got["h"].detach().cpu().double() if d["x"].dtype is F else None)
    for k, v in got.items():
        if k in want:
            ref.check(v, want[k], (what, k))
        else:
            assert v is None or not v.any(), (what, k)
    return got


@pytest.mark.parametrize("n", [8, 9, 64, 65, 511, 512, 768, 1001, 1024, 1032, 2048, 4096, 4099, 8192, 16383, 16384])
@pytest.mark.parametrize("types", ["bf16", "f32_stream", "f32"])
def test_widths(n, types):
    d, dh, dout = make(13, n, types)
    compare(d, {}, dh, dout)
    d, dh, dout = make(13, n, types, "rms", "rms", 1, bias=False)
    compare(d, dict(p=0.25, seed=7, offset=3), dh, dout)


@pytest.mark.parametrize("norm,post", list(itertools.product(["layer", "rms", None], ["layer", "rms", None])))
@pytest.mark.parametrize("types", list(TYPES))
def test_kinds(norm, post, types):
    for gate in (0, 1, 3):
        d, dh, dout = make(33, 200, types, norm, post, gate)
        compare(d, dict(x_scale=0.75, y_scale=-0.5, p=0.1, seed=2 ** 63 + 5, offset=2 ** 40 + 1), dh, dout if norm else None,
                (norm, post, gate))


@pytest.mark.parametrize("M", [1, 2, 3, 4, 5, 63, 257, 1000, 6143])
@pytest.mark.parametrize("n", [72, 1536])
def test_rows(M, n):
    d, dh, dout = make(M, n, "bf16", post="layer", gate=1)
    compare(d, {}, dh, dout)
    d, dh, dout = make(M, n, "f32")
    compare(d, {}, dh, dout)


@pytest.mark.parametrize("groups", [1, 2, 7, 70, 490])
@pytest.mark.parametrize("n", [64, 2056])
def test_gate_groups(groups, n):
    d, dh, dout = make(490, n, "bf16", "rms", None, groups)
    if groups == 1:
        d["gate"] = d["gate"].view(1, n)
    compare(d, dict(y_scale=2.0), dh, dout)


def test_one_gradient_or_the_other():
    d, dh, dout = make(40, 264, "bf16", "layer", "rms", 1)
    got = compare(d, {}, dh, None)
    assert not got["weight"].any() and not got["bias"].any()
    compare(d, {}, None, dout)
    d, dh, dout = make(40, 264, "f32")
    compare(d, {}, None, dout)


def test_reading_h_instead():
    for types, kw in (("bf16", dict(p=0.2, seed=9)), ("f32_stream", {})):
        d, dh, dout = make(60, 136, types, "layer", "rms", 2)
        c = {k: d[k].cuda() for k in NAMES if d[k] is not None}
        args = dict(post_norm="rms", post_weight=c["post_weight"], post_bias=c["post_bias"], gate=c["gate"], **kw)
        h, out, stats, post_stats = lm.add_norm(c["x"], c["y"], "layer", c["weight"], c["bias"], keep=True, **args)
        grads = (dh.cuda(), dout.cuda(), stats, post_stats)
        want = reference(d, kw, dh, dout, h.cpu().double())
        got = lm.add_norm_backward(*grads, None, c["y"], "layer", c["weight"], c["bias"], h=h, **args)
        assert sorted(got) == sorted(NAMES)
        for k, v in got.items():
            ref.check(v, want[k], k)
        # one of them alone is the same one
        for k in NAMES:
            one = lm.add_norm_backward(*grads, None, c["y"], "layer", c["weight"], c["bias"], h=h, want=(k,), **args)
            assert list(one) == [k] and torch.equal(one[k], got[k])
        with pytest.raises(ValueError):
            lm.add_norm_backward(*grads, c["x"], c["y"], "layer", c["weight"], c["bias"], h=h, **args)


def test_norm_alone():
    for types in ("bf16", "f32"):
        d, dh, dout = make(50, 328, types, with_y=False)
        compare(d, {}, dh, dout)
    # an fp32 stream normed for bf16 blocks
    d, dh, dout = make(50, 328, "f32_stream", with_y=False)
    got = step(d, {"dtype": BF}, dh, dout)
    want = reference(d, {}, dh, dout, got["h"].detach().cpu().double())
    assert got["out"].dtype is BF and got["h"].dtype is F
    for k, v in got.items():
        if v is not None:
            ref.check(v, want[k], k)


def test_same_gradient_for_both_leaves_is_not_shared_memory():
    d, dh, dout = make(20, 64, "bf16")
    x, y = (d[k].cuda().requires_grad_(True) for k in ("x", "y"))
    h, out = nn.add_norm(x, y, "layer", d["weight"].cuda(), d["bias"].cuda())
    torch.autograd.backward([h, out], [dh.cuda(), dout.cuda()])
    assert torch.equal(x.grad, y.grad)
    x.grad.zero_()
    assert y.grad.any()


def test_rows_far_from_zero():
    # a mean a thousand times the deviation: the mean is taken out before squaring
    d, dh, dout = make(21, 768, "f32", shift=2000.0)
    compare(d, {}, dh, dout)


def test_constant_and_zero_rows():
    d, dh, dout = make(6, 96, "f32", "layer", "rms")
    d["x"][:3] = 0
    d["y"][:2] = 0
    compare(d, {}, dh, dout)


def test_infinities_and_nan_stay_in_their_rows_and_what_is_dropped_does_not_count():
    d, dh, dout = make(8, 256, "bf16", gate=1)
    clean = compare(d, {}, dh, dout)
    bad = dict(d)
    bad["y"] = d["y"].clone()
    bad["y"][2, 5] = float("inf")
    bad["y"][5, 7] = float("nan")
    got = step(bad, {}, dh, dout)
    ok = [0, 1, 3, 4, 6, 7]
    for k in ("h", "out", "x", "y"):
        assert torch.equal(got[k][ok], clean[k][ok])
        assert not torch.isfinite(got[k][[2, 5]].float()).all(1).any()
    # everything dropped: y does not count, whatever it holds
    got = step(bad, dict(p=1.0), dh, dout)
    assert torch.equal(got["h"], d["x"].cuda())
    assert not got["y"].any() and not got["gate"].any()


def test_in_place_and_repeated():
    d, dh, dout = make(301, 768, "bf16", "rms", "layer")
    want = step(d, dict(p=0.2, seed=3), dh, dout)
    again = step(d, dict(p=0.2, seed=3), dh, dout)
    for k in want:
        assert want[k] is None or torch.equal(want[k], again[k])
    import paper_2312_06881_amd as dy
    c = {k: d[k].cuda() for k in NAMES if d[k] is not None}
    x, y = c["x"], c["y"]
    a = dy.AddNormArgs(301, 768, 1, dy.BF16, dy.BF16, dy.BF16, dy.NORM_RMS, dy.NORM_LAYER, 1.0, 1.0, 1e-5, 0.2, 3, 0, None,
                       x.data_ptr(), y.data_ptr(), c["weight"].data_ptr(), c["bias"].data_ptr(),
                       c["post_weight"].data_ptr(), c["post_bias"].data_ptr(), None, x.data_ptr(), y.data_ptr(), None, None)
    assert dy.dyad_add_norm_forward(a, torch.cuda.current_stream().cuda_stream) == 0
    assert torch.equal(x, want["h"]) and torch.equal(y, want["out"])


def test_inference_is_the_training_forward():
    d, _, _ = make(77, 1000, "bf16", "layer", "layer", 1)
    c = {k: d[k].cuda() for k in NAMES if d[k] is not None}
    args = dict(post_norm="layer", post_weight=c["post_weight"], post_bias=c["post_bias"], gate=c["gate"])
    with torch.no_grad():
        h0, o0 = nn.add_norm(c["x"].view(7, 11, 1000), c["y"].view(7, 11, 1000), "layer", c["weight"], c["bias"], **args)
    h1, o1 = nn.add_norm(c["x"].requires_grad_(True), c["y"], "layer", c["weight"], c["bias"], **args)
    assert h0.shape == (7, 11, 1000) and torch.equal(h0.view(77, -1), h1) and torch.equal(o0.view(77, -1), o1)


def test_against_differences():
    # a step along a random direction moves sum(h dh + out dout) by its product with the gradient
    d, dh, dout = make(9, 40, "f32", "layer", "rms", 3)
    d["gate"] = d["gate"][:3]
    v = {k: d[k].double() for k in NAMES if d[k] is not None}
    got = step(d, dict(p=0.3, seed=11), dh, dout)

    def value(at):
        r = reference({**d, **{k: t for k, t in at.items()}}, dict(p=0.3, seed=11), None, None)
        return float((r["h"][0] * dh.double()).sum() + (r["out"][0] * dout.double()).sum())

    g = torch.Generator().manual_seed(5)
    for k, t in v.items():
        e = torch.randn(t.shape, generator=g, dtype=torch.float64)
        diff = (value({**v, k: t + 1e-5 * e}) - value({**v, k: t - 1e-5 * e})) / 2e-5
        along = float((got[k].cpu().double() * e).sum())
        assert abs(diff - along) <= 1e-4 * float((got[k].cpu().double().abs() * e.abs()).sum()) + 1e-4, k


def test_empty_batch():
    d, dh, dout = make(0, 64, "bf16", "layer", "rms", 1)
    got = step(d, {}, dh, dout)
    assert got["h"].shape == (0, 64)
    for k in ("weight", "bias", "post_weight", "post_bias", "gate"):
        assert not got[k].any()


def test_module():
    torch.manual_seed(0)
    m = nn.AddNorm(96, post_norm="rms", gate=True, p=0.5, device="cuda")
    x, y = (torch.randn(2, 5, 96, device="cuda", dtype=BF) for _ in range(2))
    h, out = m(x, y)
    h2, _ = m(x, y)
    assert not torch.equal(h, h2)           # the next call's mask is another one
    m.eval()
    h, out = m(x, y)
    assert torch.equal(h, m(x, y)[0])
    want = torch.nn.functional.layer_norm(h.float(), (96,))
    # out is rounded, and so is h before torch norms it: 2^-8 of each, the norm's scale near 1
    assert (out.float() - want).abs().max() <= 2 ** -8 * want.abs().max() + 2 ** -8 * (h.float().abs().max() * 2 + 4)
    h, a = nn.AddNorm(96, "rms", device="cuda")(x)
    assert torch.equal(h, x) and a.shape == x.shape

"""What stands around the Dyad layers of a language model in training, as timed cases.

A block is y = FF(norm(x)), x <- x + y, and after the last one the loss over the vocabulary.

Kinds:
  dropout  values kept with probability 1 - p by a counter-based generator, and the gradient
  norm     h = x_scale x + y_scale gate * dropout(post(y)),  out = norm(h): a block's output joins
           the residual stream and the next block's input is normed; post is a norm of its own
           (or none), gate one vector or one a sequence (or none); with train, every gradient
  loss     softmax cross entropy of x W^T against target tokens; with train, the mean over the
           counted tokens and the gradients of x and W, else every token's loss

The generator is Philox-4x32 of ten rounds: key the seed, counter (octet, offset), 64 bits each,
octet = row * ceil(cols / 8) + col / 8.  Value j of an octet has bits 16 (j % 2) .. + 15 of word
j / 2, and is dropped where they are below t = round(65536 p); the others are scaled by
65536 / (65536 - t).
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

_TORCH = {"bf16": torch.bfloat16, "f32": torch.float32}
_BYTES = {"bf16": 2, "f32": 4}


def _dropout(name, tokens, width, p, dtype="bf16"):
    return {"name": name, "kind": "dropout", "tokens": tokens, "width": width, "p": p, "dtype": dtype}


def _norm(name, tokens, width, norm="layer", post="none", gate="none", groups=1, p=0.0, stream="bf16", dtype="bf16",
          params="bf16", x_scale=1.0, y_scale=1.0, train=True):
    return {"name": name, "kind": "norm", "tokens": tokens, "width": width, "norm": norm, "post": post, "gate": gate,
            "groups": groups, "p": p, "stream": stream, "dtype": dtype, "params": params, "x_scale": x_scale,
            "y_scale": y_scale, "train": train}


def _loss(name, tokens, width, vocab, ignored=0.0, dtype="bf16", train=True):
    return {"name": name, "kind": "loss", "tokens": tokens, "width": width, "vocab": vocab, "ignored": ignored,
            "dtype": dtype, "train": train}


def listed():
    return [
        # the embedded tokens of an OPT-125m batch, 8 sequences of 2048
        _dropout("dropout_opt125m", 16384, 768, 0.1),
        # an odd fp32 matrix
        _dropout("dropout_odd_f32", 4099, 1001, 0.25, "f32"),
        # one decoded token: the smallest call
        _norm("norm_decode", 1, 768, train=False),
        # a prompt through a wide model with norms on both sides of its blocks, no bias
        _norm("norm_wide_prompt", 2047, 8192, "rms", "rms", stream="bf16", train=False),
        # OPT-125m pretraining: dropout, residual and layer norm between two blocks
        _norm("norm_opt125m_train", 16384, 768, p=0.1),
        # a deep stack with an fp32 stream, sandwich norms, layer scale, and a residual scale
        _norm("norm_sandwich_train", 8192, 4096, "rms", "rms", "vector", stream="f32", y_scale=0.5),
        # gates that differ by sequence (7 of 571 tokens), a width of no whole vectors, fp32
        _norm("norm_gated_odd_f32", 3997, 1001, "layer", "layer", "groups", 7, 0.1, "f32", "f32", "f32"),
        # the loss of an OPT-125m batch over its vocabulary, the largest allocation of a training step
        _loss("loss_opt125m_train", 16384, 768, 50000),
        # fine tuning: half of the tokens are prompt and count for nothing; ragged everywhere
        _loss("loss_tuning_train", 3001, 1000, 50021, 0.5),
        # a wider model over a vocabulary of whole tiles
        _loss("loss_d4096_train", 4096, 4096, 32768),
        # scoring one continuation token: a stream of the weights
        _loss("loss_score_one", 1, 1024, 50000, train=False),
        # fp32, a small vocabulary
        _loss("loss_small_f32_train", 1111, 768, 5003, 0.1, "f32"),
    ]


_WIDTHS = [768, 1024, 2048, 4096]
_MAX_LOSS = 6.0 * 4096 * 4096 * 32768                      # loss_d4096_train
_MAX_NORM = 8192 * 4096


def draw(rng):
    def log(lo, hi):
        return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))

    kind = rng.choice(["dropout", "norm", "norm", "norm", "loss", "loss", "loss"])
    width = rng.choice(_WIDTHS) if rng.random() < 0.7 else log(65, 5000)
    if kind == "dropout":
        return _unnamed(_dropout("", log(16, min(16384, _MAX_NORM // width)), width, rng.choice([0.05, 0.1, 0.1, 0.25, 0.5]),
                                 rng.choice(["bf16", "bf16", "f32"])))
    if kind == "norm":
        train = rng.random() < 0.7
        stream, dtype = rng.choice([("bf16", "bf16"), ("bf16", "bf16"), ("f32", "bf16"), ("f32", "f32")])
        if rng.random() < 0.2:
            width = 8192
        tokens, groups = log(16 if train else 1, min(16384, _MAX_NORM // width)), 1
        gate = rng.choice(["none", "none", "vector", "groups"])
        if gate == "groups":
            groups = min(tokens, rng.choice([2, 3, 8, 16]))
            tokens = tokens // groups * groups
        return _unnamed(_norm("", tokens, width, rng.choice(["layer", "rms"]), rng.choice(["none", "none", "layer", "rms"]),
                              gate, groups, rng.choice([0.0, 0.1, 0.2]) if train else 0.0, stream, dtype,
                              dtype if rng.random() < 0.7 else "f32", rng.choice([1.0, 1.0, 0.75]),
                              rng.choice([1.0, 1.0, 0.5]), train))
    train = rng.random() < 0.7
    dtype = "f32" if rng.random() < 0.25 else "bf16"
    vocab = log(5000, 65000)
    if rng.random() < 0.4:
        vocab = vocab // 128 * 128
    most = _MAX_LOSS / (6.0 if train else 2.0) / width / vocab
    if dtype == "f32":
        most /= 16
    tokens = log(64 if train else 1, max(65, int(min(16384, most))))
    return _unnamed(_loss("", tokens, width, vocab, rng.choice([0.0, 0.0, 0.3]), dtype, train))


def _unnamed(case):
    del case["name"]
    return case


# ---- inputs ------------------------------------------------------------------------------

def _inputs(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    M, n = case["tokens"], case["width"]
    dt = _TORCH[case["dtype"]]

    def normal(shape, std, mean=0.0, dtype=dt):
        return (torch.randn(shape, generator=g, device="cuda") * std + mean).to(dtype)

    rng = (seed * 0x9E3779B97F4A7C15 + 12345) % 2 ** 63, seed % 1000           # the generator's seed and offset
    if case["kind"] == "dropout":
        return {"x": normal((M, n), 1.0), "dy": normal((M, n), 1.0), "rng": rng}
    if case["kind"] == "norm":
        st, pt = _TORCH[case["stream"]], _TORCH[case["params"]]
        # the stream of a trained model: a few channels much larger than the rest
        big = torch.where(torch.rand((n,), generator=g, device="cuda") < 0.01, 8.0, 1.0)
        d = {"x": (torch.randn((M, n), generator=g, device="cuda") * 2.0 * big).to(st), "y": normal((M, n), 1.0), "rng": rng,
             "dh": normal((M, n), 1.0, dtype=st), "dout": normal((M, n), 1.0)}
        d["w"] = normal((n,), 0.2, 1.0, pt)
        d["b"] = normal((n,), 0.2, 0.0, pt) if case["norm"] == "layer" else None
        d["pw"] = normal((n,), 0.2, 1.0, pt) if case["post"] != "none" else None
        d["pb"] = normal((n,), 0.2, 0.0, pt) if case["post"] == "layer" else None
        d["gate"] = None
        if case["gate"] != "none":
            d["gate"] = normal((n,) if case["gate"] == "vector" else (case["groups"], n), 0.3, 0.5, pt)
        return d
    V = case["vocab"]
    w = normal((V, n), 1.5 / math.sqrt(n))
    # frequent tokens come first, as vocabularies are sorted, and hidden states lean towards their target
    t = (float(V) ** torch.rand((M,), generator=g, device="cuda", dtype=torch.float64) - 1.0).long().clamp(0, V - 1)
    x = (torch.randn((M, n), generator=g, device="cuda") + 2.0 * w[t].float()).to(dt)
    if case["ignored"]:
        t = torch.where(torch.rand((M,), generator=g, device="cuda") < case["ignored"], -100, t)
    return {"x": x, "w": w, "t": t}


# ---- the operators in plain form: elementary operations in 32 bits -------------------------

def _mulhilo(c, k):
    """High and low 32 bits of c * k, for c of 32 bits held in 64."""
    lo, hi = (c & 0xFFFF) * k, (c >> 16) * k
    mid = (lo >> 16) + hi                                     # k < 2^32, so below 2^49
    return mid >> 16, ((mid & 0xFFFF) << 16) | (lo & 0xFFFF)


def _keep(rows, cols, p, rng):
    """Which values are kept, [rows, cols], and their scale."""
    seed, offset = rng
    octets = -(-cols // 8)
    o = torch.arange(rows * octets, device="cuda", dtype=torch.int64)
    c = [o & 0xFFFFFFFF, o >> 32, torch.full_like(o, offset & 0xFFFFFFFF), torch.full_like(o, offset >> 32)]
    k0, k1 = seed & 0xFFFFFFFF, seed >> 32
    for _ in range(10):
        h0, l0 = _mulhilo(c[0], 0xD2511F53)
        h1, l1 = _mulhilo(c[2], 0xCD9E8D57)
        c = [h1 ^ c[1] ^ k0, l1, h0 ^ c[3] ^ k1, l0]
        k0, k1 = (k0 + 0x9E3779B9) & 0xFFFFFFFF, (k1 + 0xBB67AE85) & 0xFFFFFFFF
    halves = torch.stack([v for w in c for v in (w & 0xFFFF, w >> 16)], 1).view(rows, octets * 8)[:, :cols]
    t = round(65536 * p)
    return halves >= t, 65536.0 / (65536 - t)


def _unit(v, kind, eps=1e-5):
    """v normed along its rows, without weights, and the reciprocal of what it was divided by."""
    if kind == "layer":
        v = v - v.sum(1, keepdim=True) / v.shape[1]
    r = torch.rsqrt((v * v).sum(1, keepdim=True) / v.shape[1] + eps)
    return v * r, r


def _unit_grad(du, u, r, kind):
    n = u.shape[1]
    d = du - u * ((du * u).sum(1, keepdim=True) / n)
    if kind == "layer":
        d = d - du.sum(1, keepdim=True) / n
    return d * r


def _affine(u, w, b):
    u = u * w.float()
    return u if b is None else u + b.float()


def _run_norm(case, s):
    st, dt, pt = _TORCH[case["stream"]], _TORCH[case["dtype"]], _TORCH[case["params"]]
    M, n, xs, ys = case["tokens"], case["width"], case["x_scale"], case["y_scale"]
    x, y = s["x"].float(), s["y"].float()
    z = y
    if case["post"] != "none":
        uy, ry = _unit(y, case["post"])
        z = _affine(uy, s["pw"], s["pb"])
    if case["p"]:
        keep, scale = _keep(M, n, case["p"], s["rng"])
        z = torch.where(keep, z * scale, 0.0)
    gate = None
    if s["gate"] is not None:
        gate = s["gate"].float().view(-1, 1, n).expand(-1, M // case["groups"], n).reshape(M, n)
    h = x * xs + (z if gate is None else z * gate) * ys
    uh, rh = _unit(h, case["norm"])
    out = [h.to(st), _affine(uh, s["w"], s["b"]).to(dt)]
    if not case["train"]:
        return out
    dout = s["dout"].float()
    g = s["dh"].float() + _unit_grad(dout * s["w"].float(), uh, rh, case["norm"])
    dz = g * ys
    dgate = None
    if gate is not None:
        dgate = (dz * z).view(case["groups"], -1, n).sum(1).view(s["gate"].shape)
        dz = dz * gate
    if case["p"]:
        dz = torch.where(keep, dz * scale, 0.0)
    grads = [(dout * uh).sum(0), dout.sum(0) if s["b"] is not None else None]
    dy = dz
    if case["post"] != "none":
        grads += [(dz * uy).sum(0), dz.sum(0) if s["pb"] is not None else None]
        dy = _unit_grad(dz * s["pw"].float(), uy, ry, case["post"])
    grads.append(dgate)
    return out + [(g * xs).to(st), dy.to(dt)] + [t.to(pt) for t in grads if t is not None]


def _run_loss(case, s):
    dt = _TORCH[case["dtype"]]
    x, w, t = s["x"].float(), s["w"].float(), s["t"]
    counted = t >= 0
    at = torch.where(counted, t, 0).view(-1, 1)
    z = x @ w.t()
    top = z.amax(1, keepdim=True)
    e = torch.exp(z - top)
    total = e.sum(1, keepdim=True)
    losses = torch.where(counted, (torch.log(total) + top - z.gather(1, at)).view(-1), 0.0)
    if not case["train"]:
        return losses
    count = counted.sum()
    dz = e / total
    dz.scatter_add_(1, at, torch.full_like(top, -1.0))
    dz *= (counted / count).float().view(-1, 1)
    return (losses.double().sum() / count).float(), (dz @ w).to(dt), (dz.t() @ x).to(dt)


def _run_plain(case, s):
    if case["kind"] == "norm":
        return _run_norm(case, s)
    if case["kind"] == "loss":
        return _run_loss(case, s)
    keep, scale = _keep(case["tokens"], case["width"], case["p"], s["rng"])
    return [torch.where(keep, s[k].float() * scale, 0.0).to(s[k].dtype) for k in ("x", "dy")]


# ---- a case on the GPU -----------------------------------------------------------------------

def prepare(case, seed):
    s = _inputs(case, seed)
    s["case"] = case
    if own:
        from paper_2312_06881_amd import nn  # noqa: F401  (loads the library)
        if case["kind"] == "dropout" or case["train"]:
            names = {"dropout": ["x"], "norm": ["x", "y", "w", "b", "pw", "pb", "gate"], "loss": ["x", "w"]}[case["kind"]]
            s["leaves"] = [s[k].requires_grad_(True) for k in names if s[k] is not None]
    return s


def run(state):
    case, s = state["case"], state
    if not own:
        return _run_plain(case, s)
    from paper_2312_06881_amd import nn
    if case["kind"] == "dropout":
        y = nn.dropout(s["x"], case["p"], *s["rng"])
        return [y.detach(), *torch.autograd.grad(y, s["leaves"], s["dy"])]
    if case["kind"] == "norm":
        def call():
            return nn.add_norm(s["x"], s["y"], case["norm"], s["w"], s["b"],
                               post_norm=None if case["post"] == "none" else case["post"], post_weight=s["pw"],
                               post_bias=s["pb"], gate=s["gate"], x_scale=case["x_scale"], y_scale=case["y_scale"],
                               p=case["p"], seed=s["rng"][0], offset=s["rng"][1])
        if not case["train"]:
            with torch.no_grad():
                return list(call())
        h, out = call()
        return [h.detach(), out.detach(), *torch.autograd.grad((h, out), s["leaves"], (s["dh"], s["dout"]))]
    if not case["train"]:
        with torch.no_grad():
            return nn.linear_cross_entropy(s["x"], s["w"], s["t"], reduction="none")
    loss = nn.linear_cross_entropy(s["x"], s["w"], s["t"])
    return (loss.detach(), *torch.autograd.grad(loss, s["leaves"]))


def work(case):
    M, n, e = case["tokens"], case["width"], _BYTES[case["dtype"]]
    if case["kind"] == "dropout":
        return {"bytes": 4 * e * M * n, "flops": 4.0 * M * n}
    if case["kind"] == "norm":
        vectors = 1 + (case["norm"] == "layer") + (case["post"] != "none") + (case["post"] == "layer")
        vectors += {"none": 0, "vector": 1, "groups": case["groups"]}[case["gate"]]
        rows = 2 * (e + _BYTES[case["stream"]]) * M * n          # x, y in; h, out out
        both = 2 if case["train"] else 1                         # the gradients of each
        return {"bytes": both * (rows + vectors * n * _BYTES[case["params"]]), "flops": both * 16.0 * M * n}
    V = case["vocab"]
    if not case["train"]:
        return {"bytes": e * (M + V) * n + 12 * M, "flops": 2.0 * M * n * V}
    return {"bytes": 2 * e * (M + V) * n + 8 * M + 4, "flops": 6.0 * M * n * V}


# ---- the same in 64 bits, from the definition ----------------------------------------------------

def _factors(rows, cols, p, rng):
    """0 or the scale for every value, [rows, cols] in 64 bits."""
    seed, offset = rng
    mask, s32 = np.uint64(0xFFFFFFFF), np.uint64(32)
    octets = (cols + 7) // 8
    n = np.arange(rows * octets, dtype=np.uint64)
    x0, x1 = n & mask, n >> s32
    x2 = np.full_like(n, offset % 2 ** 32)
    x3 = np.full_like(n, offset // 2 ** 32)
    for r in range(10):
        a, b = np.uint64(0xD2511F53) * x0, np.uint64(0xCD9E8D57) * x2
        ka = np.uint64((seed % 2 ** 32 + r * 0x9E3779B9) % 2 ** 32)
        kb = np.uint64((seed // 2 ** 32 + r * 0xBB67AE85) % 2 ** 32)
        x0, x1, x2, x3 = (b >> s32) ^ x1 ^ ka, b & mask, (a >> s32) ^ x3 ^ kb, a & mask
    words = np.stack([x0, x1, x2, x3], axis=1).astype("<u4")
    u = words.view("<u2").reshape(rows, octets * 8)[:, :cols].astype(np.int32)
    t = int(np.rint(p * 65536))
    return torch.from_numpy(u >= t).cuda().double() * (65536 / (65536 - t))


class _Normed:
    """(v - mean) / deviation along the rows (layer) or v / root mean square (rms), and its gradient."""

    def __init__(self, v, kind):
        self.centred = kind == "layer"
        c = v - v.mean(1, keepdim=True) if self.centred else v
        self.s = (c.square().mean(1, keepdim=True) + 1e-5).sqrt()
        self.value = c / self.s

    def grad(self, d):
        # of v_i / s: d_i / s - v_i (sum_j d_j v_j) / (n s^3), centred where the mean was taken out
        d = (d - self.value * (d * self.value).mean(1, keepdim=True)) / self.s
        return d - d.mean(1, keepdim=True) if self.centred else d


def _exact_norm(case, s):
    M, n, B = case["tokens"], case["width"], case["groups"]
    v = {k: None if t is None or k == "rng" else t.double() for k, t in s.items()}
    factor = _factors(M, n, case["p"], s["rng"]) if case["p"] else 1.0
    gate = 1.0
    if v["gate"] is not None:
        gate = v["gate"].view(B, n).repeat_interleave(M // B, 0)
    inner = _Normed(v["y"], case["post"]) if case["post"] != "none" else None
    z = v["y"]
    if inner:
        z = inner.value * v["pw"] + (0.0 if v["pb"] is None else v["pb"])
    h = case["x_scale"] * v["x"] + case["y_scale"] * factor * gate * z
    outer = _Normed(h, case["norm"])
    out = [h, outer.value * v["w"] + (0.0 if v["b"] is None else v["b"])]
    if not case["train"]:
        return out
    dh = v["dh"] + outer.grad(v["dout"] * v["w"])
    dz = dh * case["y_scale"] * factor * gate
    out += [dh * case["x_scale"], inner.grad(dz * v["pw"]) if inner else dz, (v["dout"] * outer.value).sum(0)]
    if v["b"] is not None:
        out.append(v["dout"].sum(0))
    if inner:
        out.append((dz * inner.value).sum(0))
        if v["pb"] is not None:
            out.append(dz.sum(0))
    if v["gate"] is not None:
        out.append((dh * case["y_scale"] * factor * z).unflatten(0, (B, -1)).sum(1).view(s["gate"].shape))
    return out


def exact(case, seed):
    s = _inputs(case, seed)
    if case["kind"] == "dropout":
        f = _factors(case["tokens"], case["width"], case["p"], s["rng"])
        return [s["x"].double() * f, s["dy"].double() * f]
    if case["kind"] == "norm":
        return _exact_norm(case, s)
    w, t = s["w"].double(), s["t"]
    used = (t != -100).nonzero().view(-1)
    losses = torch.zeros(t.shape[0], dtype=torch.float64, device="cuda")
    dx = torch.zeros(s["x"].shape, dtype=torch.float64, device="cuda")
    dw = torch.zeros_like(w)
    for rows in used.split(2048):
        x = s["x"][rows].double()
        z = x @ w.t()
        lse = torch.logsumexp(z, 1)
        losses[rows] = lse - z[torch.arange(len(rows), device="cuda"), t[rows]]
        if case["train"]:
            p = torch.exp(z - lse[:, None])
            p[torch.arange(len(rows), device="cuda"), t[rows]] -= 1.0
            p /= len(used)
            dx[rows] = p @ w
            dw += p.t().contiguous() @ x
    if not case["train"]:
        return losses
    return losses.sum() / len(used), dx, dw

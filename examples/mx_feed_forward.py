"""A feed-forward block trained on 8-bit activation checkpoints and served in 4 bits.

Trains ``DyadFF(stash="mx8")`` to follow a fixed dense block on synthetic tokens, quantises
its weights with ``MX4DyadFF`` and runs a prompt and then single tokens through it.

    python examples/mx_feed_forward.py [--d 768 --ffn 3072 --n-dyad 4 --variant IT --tokens 4096 --steps 200]
"""
import argparse
import os
import sys

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import torch

from paper_2312_06881_amd.nn import DyadFF, MX4DyadFF


def kept_bytes(block, x):
    """Bytes that one forward pass keeps for its backward pass, parameters aside."""
    own = {p.data_ptr() for p in block.parameters()}
    sizes = []

    def pack(t):
        if t.data_ptr() not in own:
            sizes.append(t.nbytes)
        return t

    with torch.autograd.graph.saved_tensors_hooks(pack, lambda t: t):
        block(x)
    return sum(sizes)


def run(d=768, ffn=3072, n_dyad=4, variant="IT", tokens=4096, steps=200, seed=0):
    torch.manual_seed(seed)
    dev = "cuda"
    teacher = torch.nn.Sequential(torch.nn.Linear(d, d), torch.nn.Tanh()).to(dev)
    block = DyadFF(d, ffn, n_dyad, variant, device=dev, stash="mx8")
    plain = DyadFF(d, ffn, n_dyad, variant, device=dev)
    optimizer = torch.optim.AdamW(block.parameters(), lr=2e-3)
    losses = []
    for _ in range(steps):
        x = torch.randn(tokens, d, device=dev)
        with torch.no_grad():
            target = teacher(x)
        loss = (block(x.bfloat16()).float() - target).square().mean()
        optimizer.zero_grad()
        loss.backward()
        optimizer.step()
        losses.append(loss.detach())
    x = torch.randn(tokens, d, device=dev).bfloat16()
    result = {"loss": (float(losses[0]), float(losses[-1])),
              "kept": (kept_bytes(block, x.requires_grad_(True)), kept_bytes(plain, x))}
    served = MX4DyadFF(block)
    with torch.no_grad():
        prompt = x.detach()
        full, y = block(prompt), served(prompt)
        one = torch.cat([served(prompt[i:i + 1]) for i in range(8)])
    result["fp4"] = float((y.float() - full.float()).norm() / full.float().norm())
    result["single"] = float((one.float() - y[:8].float()).abs().max())
    result["weights"] = (sum(p.nbytes for p in block.parameters()), sum(b.nbytes for b in served.buffers()))
    return result


def main():
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    for name, value in (("d", 768), ("ffn", 3072), ("n-dyad", 4), ("tokens", 4096), ("steps", 200)):
        ap.add_argument(f"--{name}", type=int, default=value)
    ap.add_argument("--variant", choices=("IT", "OT", "DT"), default="IT")
    r = run(**vars(ap.parse_args()))
    print("training loss %.4f -> %.4f" % r["loss"])
    print("kept for the backward pass: %d bytes in 8 bits, %d in bf16" % r["kept"])
    print("weights: %d bytes in bf16, %d in fp4" % r["weights"])
    print("fp4 against bf16 outputs: %.3f of their norm; one token at a time against the prompt: at most %.2g" %
          (r["fp4"], r["single"]))


if __name__ == "__main__":
    main()

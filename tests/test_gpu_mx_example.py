"""The feed-forward example end to end: it learns on 8-bit checkpoints, and the fp4 block follows it."""
import pytest

import paper_2312_06881_amd as dy
from examples.mx_feed_forward import run

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("variant", ("IT", "OT", "DT"))
def test_example(variant):
    print("CASE example", variant, flush=True)
    r = run(d=256, ffn=1024, n_dyad=4, variant=variant, tokens=512, steps=60)
    first, last = r["loss"]
    assert last < 0.7 * first
    # x and h in 8 bits and a scale for 32, against x, h and GELU(h) in 16
    assert r["kept"][0] == 512 * (256 + 1024) * 33 // 32
    assert r["kept"][1] >= 512 * 2 * (256 + 2 * 1024)
    # fp4 blocks in whole steps of 128 reduction indices, and the biases
    v = dy.VARIANTS[variant]
    assert r["weights"][1] == dy.dyad_mx4_weight_bytes(v, 256, 1024, 4) + dy.dyad_mx4_weight_bytes(v, 1024, 256, 4) + 2 * 1280
    assert r["weights"][1] < 0.5 * r["weights"][0]
    # elements of 4 bits: steps of up to a third of the value in weights and inputs of two layers
    assert r["fp4"] < 0.5
    # a token alone and in the prompt: one bf16 rounding and fp32 sums in another order, and where
    # those move a hidden value across a rounding boundary of fp4, one of 1024 terms by a step
    assert r["single"] < 0.05

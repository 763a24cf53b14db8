"""fp32 passes on tiles of every size: the tile depends on the batch, a token's sums do not."""
import pytest
import torch

import paper_2312_06881_amd as dy

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("variant", ["IT", "OT", "DT"])
@pytest.mark.parametrize("n_in,n_out,D", [(256, 1024, 4), (1024, 256, 2), (384, 160, 8)])
def test_rows_do_not_depend_on_the_batch(variant, n_in, n_out, D):
    g = torch.Generator(device="cuda").manual_seed(7)
    big = 6000
    x = torch.randn((big, n_in), generator=g, device="cuda")
    dz = torch.randn((big, n_out), generator=g, device="cuda")
    w1, w2 = torch.randn((2, D, n_out // D, n_in // D), generator=g, device="cuda") * 0.05
    b = torch.randn((n_out,), generator=g, device="cuda")
    y = dy.forward(x, w1, w2, b, variant, act="gelu")
    dx = dy.backward_dx(dz, w1, w2, variant)
    for M in (1, 33, 200, 700, 2500):
        assert torch.equal(dy.forward(x[:M], w1, w2, b, variant, act="gelu"), y[:M])
        assert torch.equal(dy.backward_dx(dz[:M], w1, w2, variant), dx[:M])


@pytest.mark.parametrize("variant", ["IT", "OT", "DT"])
@pytest.mark.parametrize("n_in,n_out,D,M", [(256, 1024, 4, 200), (1024, 256, 2, 1100), (384, 160, 8, 65),
                                            (2048, 4096, 2, 70)])
def test_weight_gradient(variant, n_in, n_out, D, M):
    g = torch.Generator(device="cuda").manual_seed(8)
    x = torch.randn((M, n_in), generator=g, device="cuda")
    dz = torch.randn((M, n_out), generator=g, device="cuda")
    got = dy.backward_dw(dz, x, D, variant)
    G = dz.double().t() @ x.double()
    i = torch.arange(D, device="cuda").view(D, 1, 1)
    j = torch.arange(n_out // D, device="cuda").view(1, -1, 1)
    k = torch.arange(n_in // D, device="cuda").view(1, 1, -1)
    one = G[i * (n_out // D) + j, i * (n_in // D) + k]
    two = G[j * D + i if variant in ("OT", "DT") else i * (n_out // D) + j,
            k * D + i if variant in ("IT", "DT") else i * (n_in // D) + k]
    # a sum of M products of unit normals, each addition rounded: M * 2^-24 of sqrt(M) and a margin of 4
    bound = 4 * M * 2.0 ** -24 * M ** 0.5
    for a, e in zip(got, (one, two, dz.double().sum(0))):
        assert (a.double() - e).abs().max().item() <= bound

"""Dropout on the GPU: the mask is the generator's, values are scaled and rounded once."""
import pytest
import torch

from tests import lm_reference as ref
from paper_2312_06881_amd import lm, nn

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("shape", [(1,), (7,), (8,), (1, 1), (3, 5, 9), (64, 768), (129, 1001), (4099, 33)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("p", [0.0, 0.1, 0.5, 1.0])
def test_values(shape, dtype, p):
    g = torch.Generator().manual_seed(len(shape))
    x = torch.randn(shape, generator=g).to(dtype)
    cols = shape[-1]
    kept, scale = ref.keep_mask(x.numel() // cols, cols, p, 2 ** 64 - 3, 2 ** 33 + 7)
    want = (torch.where(kept, x.view(-1, cols).float() * torch.tensor(scale, dtype=torch.float32), 0.0)).to(dtype).view(shape)
    a = x.cuda().requires_grad_(True)
    y = nn.dropout(a, p, 2 ** 64 - 3, 2 ** 33 + 7)
    assert torch.equal(y.cpu(), want)
    dx, = torch.autograd.grad(y, a, torch.ones_like(y))
    ones = torch.where(kept, torch.tensor(scale, dtype=torch.float32), 0.0).to(dtype).view(shape)
    assert torch.equal(dx.cpu(), ones)


def test_scalar_and_empty():
    assert nn.dropout(torch.ones((), device="cuda"), 0.0, 1).item() == 1.0
    assert nn.dropout(torch.ones((0, 4), device="cuda"), 0.5, 1).shape == (0, 4)
    x = torch.ones(4, device="cuda")
    assert nn.dropout(x, 0.5, 1, training=False) is x


def test_dropped_values_do_not_count():
    x = torch.full((64, 64), float("nan"), device="cuda")
    kept, _ = ref.keep_mask(64, 64, 0.5, 9, 0)
    assert torch.equal(torch.isnan(lm.dropout(x, 0.5, 9)).cpu(), kept)


def test_strided_input_and_in_place():
    import paper_2312_06881_amd as dy
    x = torch.randn(96, 40, device="cuda").t()
    assert torch.equal(nn.dropout(x, 0.3, 4), lm.dropout(x.contiguous(), 0.3, 4))
    y = x.contiguous()
    want = lm.dropout(y, 0.3, 4)
    assert dy.dyad_dropout(40, 96, dy.F32, y.data_ptr(), 0.3, 4, 0, None, y.data_ptr(),
                           torch.cuda.current_stream().cuda_stream) == 0
    assert torch.equal(y, want)


def test_offset_on_the_device():
    x = torch.randn(50, 72, device="cuda", dtype=torch.bfloat16)
    off = torch.tensor([12345678901], device="cuda")
    assert torch.equal(lm.dropout(x, 0.2, 4, off), lm.dropout(x, 0.2, 4, 12345678901))
    a = x.clone().requires_grad_(True)
    y = nn.dropout(a, 0.2, 4, off)
    off += 1
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.sum().backward()                 # it would draw another mask


def test_replays_draw_other_masks():
    m = nn.Dropout(0.5, seed=77, capturable=True, device="cuda")
    x = torch.ones(33, 65, device="cuda")
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        m(x)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            y = m(x)
    for k in range(1, 5):
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, lm.dropout(x, 0.5, 77, k))
        lm.dropout(x, 0.5, 1)              # eager work in between


def test_double_backward_is_refused():
    x = torch.randn(4, 8, device="cuda", requires_grad=True)
    g, = torch.autograd.grad(nn.dropout(x, 0.5, 1).square().sum(), x, create_graph=True)
    with pytest.raises(RuntimeError):
        g.sum().backward()

"""Captured forward and backward passes beside graphs from outside of the capture."""
import pytest
import torch

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def tsr():
    import paper_2602_08007_b200 as t
    return t


def normal(*shape, seed=1):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn(*shape, generator=gen, device="cuda")


def test_a_cast_weight_is_seen(tsr):
    """The leaf is the FP32 parameter; the layer gets its BF16 image, a new tensor each time."""
    x, w = normal(64, 32).to(BF), normal(48, 32, seed=2).requires_grad_()
    eager = tsr.linear(x, w.to(BF)).sum()
    g = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with pytest.raises(RuntimeError, match="still alive"):
        with torch.cuda.graph(g):
            tsr.linear(x, w.to(BF)).sum().backward()
    g.reset()
    eager.backward()
    first = w.grad.clone()
    del eager
    w.grad = None
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        tsr.linear(x, w.to(BF)).sum().backward()
    g.replay()
    torch.cuda.synchronize()
    assert torch.equal(w.grad, first)
    g.reset()

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


def test_a_warm_up_on_a_side_stream_may_live_on(tsr):
    """The usual order: warm-up steps on a side stream, whose last outputs are still held, then the capture; the replay's gradients are those of the formula."""
    x, w, nw = normal(64, 32), normal(48, 32, seed=2).requires_grad_(), normal(32, seed=3).requires_grad_()

    def step():
        return tsr.linear(tsr.rms_norm(x, nw), w, activation="silu").square().sum()

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for _ in range(3):
            w.grad = nw.grad = None
            loss = step()
            loss.backward()
        want = [w.grad.clone(), nw.grad.clone()]
    torch.cuda.current_stream().wait_stream(side)
    w.grad = nw.grad = None
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step().backward()
    g.replay()
    torch.cuda.synchronize()
    assert loss.grad_fn is not None and torch.equal(w.grad, want[0]) and torch.equal(nw.grad, want[1])
    g.reset()

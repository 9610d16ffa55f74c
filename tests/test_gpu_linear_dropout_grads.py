"""Gradients of a layer with dropout and no activation: which entries fall is decided in dz, the factor is applied to the results, so that BF16 operands are the
upstream gradients themselves."""
import pytest
import torch

import layer_model as lm
import test_gpu_linear as tl

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def tsr():
    import paper_2602_08007_b200 as t
    return t


@pytest.mark.parametrize("p", [0.1, 0.37])
@pytest.mark.parametrize("accumulate", [False, True])
@pytest.mark.parametrize("dt", [BF, F32])
@pytest.mark.parametrize("T,I,O", [(40, 24, 16), (200, 160, 328), (65, 77, 91), (3000, 512, 512), (20000, 64, 128)])
def test_products_of_what_is_kept(tsr, T, I, O, dt, accumulate, p):
    """Bounds of the products alone and of one FP32 multiplication, with no rounding of dz; column sums of at most 2^9 additions on any path."""
    x, w, dy = tl.make((T, I), dt, 1), tl.make((O, I), dt, 2, 0.1), tl.make((T, O), dt, 3)
    g = tl.make((O, I), F32, 4) if accumulate else torch.full((O, I), float("nan"), device="cuda")
    gb = tl.make((1, O), F32, 5)[0].contiguous() if accumulate else torch.full((O,), float("nan"), device="cuda")
    g0, gb0 = (g.double(), gb.double()) if accumulate else (0.0, 0.0)
    d = tsr.Dropout(p, 77, 5)
    dx, dw, db = tsr.linear_backward(dy, x, w, dropout=d, dweight=g, dbias=gb, accumulate=accumulate)
    dz = lm.drop(dy.double(), d)
    for got, a, b, old in ((dx, dz, w.double().t(), 0.0), (dw, dz.t(), x.double().t(), g0)):
        want = a @ b.t()
        lm.close(got, want + old, lm.product_slack(a, b, dt) + 2.0 ** -23 * (want.abs() + (want + old).abs()))
    lm.close(db, dz.sum(0) + gb0, 2.0 ** -15 * dz.abs().sum(0) + 2.0 ** -23 * (dz.sum(0) + gb0).abs())


@pytest.mark.parametrize("dt", [BF, F32])
def test_everything_falls(tsr, dt):
    x, w, dy = tl.make((50, 24), dt, 1), tl.make((16, 24), dt, 2), tl.make((50, 16), dt, 3)
    dx, dw, db = tsr.linear_backward(dy, x, w, dropout=tsr.Dropout(1.0, 3), dbias=torch.empty(16, device="cuda"))
    assert not dx.any() and not dw.any() and not db.any()

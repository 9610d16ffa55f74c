"""FP32 layers beyond the sizes of their results: infinities."""
import pytest
import torch

import layer_model as lm

pytestmark = pytest.mark.gpu
F32, BF = torch.float32, torch.bfloat16


@pytest.fixture(scope="module")
def tsr():
    import paper_2602_08007_b200 as t
    return t


def normal(*shape, seed=1, sigma=1.0):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn(*shape, generator=gen, device="cuda") * sigma


@pytest.mark.parametrize("T,I,O", [(1, 72, 96), (8, 72, 96), (60, 72, 96), (65, 72, 96), (150, 73, 97), (300, 5000, 64), (2500, 512, 1376)])
def test_infinities(tsr, T, I, O):
    """An infinity comes out as the formula has it, for any number of rows: infinite against weights that are not zero, whatever bits these have, NaN against
    zeros and infinities of the other sign."""
    inf = float("inf")
    x, w = normal(T, I, seed=1), normal(O, I, seed=2)
    w[::2] = w[::2].to(BF).float()            # the lower parts of these are zero
    w[5, 3] = 0.0
    w[6, 7] = -inf
    rows = sorted({0, T // 2, T - 1})
    for i, r in enumerate(rows):
        x[r, 3] = inf if i % 2 == 0 else -inf
    x[rows[-1], 7] = inf
    x[rows[0], I - 1] = float("nan") if T > 100 else inf
    want = x.double() @ w.double().t()
    y, _ = tsr.linear_forward(x, w)
    bad = ~torch.isfinite(want)
    assert torch.equal(torch.isnan(y), torch.isnan(want)) and torch.equal(y[bad & ~torch.isnan(want)].double(), want[bad & ~torch.isnan(want)])
    if not bad.all():
        assert torch.isfinite(y[~bad]).all() and float((y.double() - want)[~bad].abs().max()) <= 2.0 ** -16 * float(want[~bad].abs().max())
    # backward: x as the gradient of a layer with as many outputs as x has columns
    g = w.t().contiguous()                     # (I, O)
    dx, _, _ = tsr.linear_backward(x, None, g, want_dweight=False)
    assert torch.equal(torch.isnan(dx), torch.isnan(want)) and torch.equal(dx[bad & ~torch.isnan(want)].double(), want[bad & ~torch.isnan(want)])
    up = normal(T, O, seed=3)
    up[::2] = up[::2].to(BF).float()
    _, dw, _ = tsr.linear_backward(up, x, torch.zeros(O, I, device="cuda"), want_dx=False)
    want = up.double().t() @ x.double()
    bad = ~torch.isfinite(want)
    assert torch.equal(torch.isnan(dw), torch.isnan(want)) and torch.equal(dw[bad & ~torch.isnan(want)].double(), want[bad & ~torch.isnan(want)])
    assert tsr.layer_poll_status() == tsr.TSR_OK

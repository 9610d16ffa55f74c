"""Activations of FP32 layers and their slopes, on every way through a layer: near the formula, and at values far out."""
import math

import pytest
import torch

import layer_model as lm

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def tsr():
    import paper_2602_08007_b200 as t
    return t


def plain(kind, z):
    if kind == "gelu":
        return 0.5 * z * (1.0 + torch.erf(z * math.sqrt(0.5)))
    if kind == "gelu_tanh":
        return 0.5 * z * (1.0 + torch.tanh(math.sqrt(2.0 / math.pi) * (z + 0.044715 * z * z * z)))
    return z / (1.0 + torch.exp(-z))


def plain_slope(kind, z):
    if kind == "gelu":
        return 0.5 * (1.0 + torch.erf(z * math.sqrt(0.5))) + z * torch.exp(-0.5 * z * z) / math.sqrt(2.0 * math.pi)
    if kind == "gelu_tanh":
        c = math.sqrt(2.0 / math.pi)
        t = torch.tanh(c * (z + 0.044715 * z * z * z))
        return 0.5 * (1.0 + t) + 0.5 * z * (1.0 - t * t) * c * (1.0 + 3 * 0.044715 * z * z)
    t = 1.0 / (1.0 + torch.exp(-z))
    return t * (1.0 + z * (1.0 - t))


def rms(got, want):
    return float(((got.double() - want) / want).square().mean().sqrt())


# a row each (few-row kernel), one launch of tiles, split K with the epilogue in the launch after it
@pytest.mark.parametrize("route", ["few", "tiles", "split"])
@pytest.mark.parametrize("kind", ["gelu", "gelu_tanh", "silu"])
def test_activations_are_as_near_as_the_plain_form(tsr, kind, route):
    """z comes through the product exactly (one entry of K, a weight of one).  Relative errors, root of the mean square, against the FP32 formula in
    elementary operations: half as much again at most, over [-1, 1]; SiLU far below zero too, where expf is within 2 units of the last place
    (2^-22), the sum and the quotient within half of one each: 3 x 2^-23 (an exponential of 1.44 z in FP32 would be off by z 2^-24)."""
    T, O = {"few": (8, 500), "tiles": (500, 300), "split": (128, 64)}[route]
    z = torch.linspace(-1, 1, T * O, device="cuda")
    z[z.abs() < 1e-3] = 0.5

    def through(z):
        K = 4096 if route == "split" else T
        x, w = torch.zeros(T, K, device="cuda"), torch.zeros(O, K, device="cuda")
        x[torch.arange(T), torch.arange(T)] = 1.0
        w[:, :T] = z.view(T, O).t()
        y, pre = tsr.linear_forward(x, w, activation=kind, keep_pre=True)
        assert torch.equal(pre.view(-1), z)
        return y.view(-1)

    want = lm.act(kind, z.double())
    assert rms(through(z), want) <= 1.5 * rms(plain(kind, z), want)
    if kind == "silu":
        z = torch.linspace(-80, -1, T * O, device="cuda")
        want = lm.act(kind, z.double())
        assert float(((through(z).double() - want) / want).abs().max()) <= 3 * 2.0 ** -23


@pytest.mark.parametrize("kind", ["gelu", "gelu_tanh", "silu"])
def test_slopes_are_as_near_as_the_plain_form(tsr, kind):
    """The bias's gradient of one row with an upstream gradient of one is the slope itself."""
    z = torch.linspace(-0.5, 2, 20001, device="cuda").view(1, -1)
    ones = torch.ones_like(z)
    _, _, db = tsr.linear_backward(ones, None, torch.zeros(20001, 1, device="cuda"), pre=z, activation=kind, dbias=torch.empty(20001, device="cuda"), want_dx=False, want_dweight=False)
    want = lm.slope(kind, z.double()).view(-1)
    assert rms(db, want) <= 1.5 * rms(plain_slope(kind, z).view(-1), want)


@pytest.mark.parametrize("dt", [F32, BF])
@pytest.mark.parametrize("route", ["few", "tiles", "split"])
@pytest.mark.parametrize("kind", lm.ACTS)
def test_values_far_out(tsr, kind, route, dt):
    """Large values, infinities and NaN are the formula's: zero below, the value itself above, NaN at minus infinity (zero times it; ReLU: zero).  Slopes there are
    zero and one, and NaN at NaN."""
    far = torch.tensor([1e30, -1e30, 1e5, -1e5, 100.0, -100.0, 30.0, -30.0, float("inf"), float("-inf"), float("nan"), 0.0], device="cuda")
    T, K = {"few": (4, 16), "tiles": (200, 16), "split": (128, 4096)}[route]
    x, w = torch.zeros(T, K, device="cuda", dtype=dt), torch.zeros(64, K, device="cuda", dtype=dt)
    b = far.repeat(6)[:64].contiguous()
    y, _ = tsr.linear_forward(x, w, b, activation=kind)
    want = lm.act(kind, b.double()).expand(T, 64)
    lm.close(y, want, 2.0 ** -18 * torch.nan_to_num(want.abs(), 0.0, 0.0, 0.0))
    pre = b.to(dt).expand(T, 64).contiguous()
    _, _, db = tsr.linear_backward(torch.ones(T, 64, device="cuda", dtype=dt), None, w, pre=pre, activation=kind, dbias=torch.empty(64, device="cuda"), want_dx=False, want_dweight=False)
    z = pre[0].double()
    slope = torch.where(torch.isinf(z), (z > 0).double(), lm.slope(kind, z.clamp(-1e5, 1e5))) if kind != "none" else torch.ones_like(z)
    if kind != "none":
        slope = torch.where(torch.isnan(z), z, slope)
    lm.close(db, slope * T, 2.0 ** -18 * torch.nan_to_num(slope * T).abs())

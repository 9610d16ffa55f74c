"""Stochastic rounding of BF16 parameters in dense plans against its definition (GPU)."""
import numpy as np
import pytest
import torch

import dense_model as dm
from dense_model import f32

pytestmark = pytest.mark.gpu

F8 = torch.float8_e4m3fn
NAN, INF = float("nan"), float("inf")


@pytest.fixture(scope="module")
def tsr():
    import paper_2602_08007_b200 as t
    return t


def rand(n, seed, scale=1.0):
    return torch.randn(n, generator=torch.Generator().manual_seed(seed)) * scale


def words16(n, seed, t, tensor):
    """The 16 random bits of each element of a BF16 parameter."""
    k1, k2 = dm.keys(seed, t, tensor)
    e = np.arange(n, dtype=np.uint64)
    w = dm.random_words((e >> 1).astype(np.uint32), k1 ^ 0x5BD1E995, k2)
    return np.where(e & 1, w >> 16, w & 0xFFFF).astype(np.uint32)


def cut(x, u):
    """FP32 values with random bits u added below BF16's and cut off."""
    return ((x.astype(np.float32).view(np.uint32) + u) & np.uint32(0xFFFF0000)).view(np.float32)


def placed(x, rows, cols, pitch, shift):
    """x as a rows x cols matrix with `pitch` elements between its rows, `shift` elements into its buffer."""
    ld = cols + pitch
    buf = torch.zeros(shift + rows * ld, dtype=x.dtype, device="cuda")
    view = torch.as_strided(buf, (rows, cols), (ld, 1), shift)
    view.copy_(x.view(rows, cols))
    return view


SHAPES = [(1, 5000, 0), (10, 500, 0), (10, 500, 3), (125, 40, 1)]


@pytest.mark.parametrize("shift", [0, 1])
@pytest.mark.parametrize("kind", [torch.float32, F8])
@pytest.mark.parametrize("rows,cols,pitch", SHAPES)
def test_bad_parameters_leave_the_others_bits_alone(tsr, rows, cols, pitch, kind, shift):
    """Without a gradient a step multiplies by 1 - lr wd.  Whatever stands beside it, a finite parameter is rounded by its own
    word; an infinite one and a NaN stay what they are."""
    n, seed, t = rows * cols, 99, 4
    p = rand(n, 1).bfloat16()
    bad = torch.arange(n) % 37 == 5
    p[bad] = torch.tensor([NAN, INF, -INF, -NAN]).bfloat16().repeat(n)[:int(bad.sum())]
    h = dict(lr=f32(2e-3), wd=f32(0.3))
    x, g = placed(p, rows, cols, pitch, shift), placed(torch.zeros(n, dtype=torch.bfloat16), rows, cols, pitch, shift)
    plan = tsr.DensePlan([x], [g], state_dtype=kind)
    plan.step(tsr.make_hyper(t, lr=h["lr"], beta2=0.99, eps=1e30, weight_decay=h["wd"]), rounding=1, seed=seed)
    F = np.float32
    decay = F(1) - F(h["lr"]) * F(h["wd"])
    with np.errstate(invalid="ignore"):
        want = cut(p.float().numpy() * decay, words16(n, seed, t, 0))
    got, bad, start = x.float().cpu().numpy().reshape(-1), bad.numpy(), p.float().numpy()
    assert np.array_equal(got[~bad], want[~bad])
    assert np.array_equal(np.isnan(got), np.isnan(start))
    assert np.array_equal(got[np.isinf(start)], start[np.isinf(start)])


@pytest.mark.parametrize("kind", [torch.float32, F8])
@pytest.mark.parametrize("bad", [NAN, INF])
def test_a_bad_gradient_reaches_its_own_parameter_alone(tsr, bad, kind):
    n, at = 3000, 1234
    out = []
    for poison in (False, True):
        p, g = rand(n, 1).bfloat16().cuda(), rand(n, 2).bfloat16().cuda()
        if poison:
            g[at] = bad
        plan = tsr.DensePlan([p], [g], state_dtype=kind)
        plan.step(tsr.make_hyper(1), rounding=1, seed=7)
        out.append(p.float().cpu())
    same = torch.arange(n) != at
    assert torch.equal(out[0][same], out[1][same]) and not torch.isfinite(out[1][at])


@pytest.mark.parametrize("shift", [0, 1])
@pytest.mark.parametrize("kind", [torch.float32, F8])
@pytest.mark.parametrize("gd", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rows,cols,pitch", SHAPES)
def test_parameters_are_cut_with_their_own_words(tsr, rows, cols, pitch, gd, kind, shift):
    """A whole step: the FP32 result is within the error bound of the definition in 64 bits, and adding a parameter's own word
    and cutting is monotonous in magnitude, so what is stored lies between the cut ends of that interval."""
    n, seed, t = rows * cols, 1 << 40 | 12345, 3
    h = dict(lr=f32(2e-3), beta1=f32(0.9), beta2=f32(0.99), eps=f32(1e-8), wd=f32(0.1), t=t)
    p = rand(n, 1, 0.02).bfloat16()
    g = (rand(n, 2) * torch.exp(2 * rand(n, 3) - 6)).to(gd)
    xs, gs = ([placed(p, rows, cols, pitch, shift) for _ in (0, 1)], [placed(x, rows, cols, pitch, shift) for x in (g, g)])
    plan = tsr.DensePlan(xs, gs, state_dtype=kind)
    hy = lambda k: tsr.make_hyper(k, lr=h["lr"], beta1=h["beta1"], beta2=h["beta2"], eps=h["eps"], weight_decay=h["wd"])  # noqa: E731
    plan.step(hy(2))       # moments that are not zero
    before = [x.double().cpu().numpy().reshape(-1) for x in xs]
    old = [[y.float().double().cpu().numpy() for y in s] for s in plan.states]
    plan.step(hy(t), rounding=1, seed=seed)
    for i in (0, 1):
        m, v = old[i][:2]
        if kind == F8:
            scale = np.repeat(old[i][2].reshape(-1, 2), dm.BLOCK, axis=0)[:n]
            m, v = m * scale[:, 0], (v * scale[:, 1]) ** 2
        p1, _, _, tol, _, _ = dm.step64(before[i], g.double().numpy(), m, v, h)
        u = words16(n, seed, t, i)
        low = cut(np.maximum(np.abs(p1) - tol * (1 + 1e-6), 0.0), u)
        high = cut(np.abs(p1) + tol * (1 + 1e-6), u)
        got = xs[i].float().cpu().numpy().reshape(-1)
        sure = np.abs(p1) > tol
        assert np.all(np.signbit(got[sure]) == np.signbit(p1[sure]))
        assert np.all((np.abs(got) >= low) & (np.abs(got) <= high))

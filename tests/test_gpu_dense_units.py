"""Dense plans with many blocks to a warp (millions of elements): every path's loop over its units, ring refills and row
advances included, against plans so small that a warp has one block, and against the model on sampled blocks (GPU)."""
import math

import numpy as np
import pytest
import torch

import dense_model as dm
from dense_model import BLOCK, E4M3, U24, f32

pytestmark = pytest.mark.gpu

F8 = torch.float8_e4m3fn
DT = {"f32": torch.float32, "bf16": torch.bfloat16}
HYPER = dict(lr=f32(2e-3), beta1=f32(0.9), beta2=f32(0.99), eps=f32(1e-8), wd=f32(0.1))
ROWS, COLS = 2101, 4290          # 9 M elements: eight blocks a warp where everything is aligned, four elsewhere
N = ROWS * COLS
PIECE = 1000 * BLOCK             # one block a warp
LAYOUTS = {"plain": (0, 0), "shifted": (0, 1), "pitched": (6, 0), "pitched and shifted": (3, 1)}


@pytest.fixture(scope="module")
def tsr():
    import paper_2602_08007_b200 as t
    return t


def hyper(tsr, t):
    return tsr.make_hyper(t, lr=HYPER["lr"], beta1=HYPER["beta1"], beta2=HYPER["beta2"], eps=HYPER["eps"], weight_decay=HYPER["wd"])


def rand(n, seed, scale=1.0):
    return torch.randn(n, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda") * scale


def gradient(n, seed):
    g = rand(n, seed) * torch.exp(2 * rand(n, seed + 1) - 6)
    g[BLOCK:2 * BLOCK] = 0
    return g


def placed(x, layout, rows=ROWS, cols=COLS):
    pitch, shift = LAYOUTS[layout]
    buf = torch.full((shift + rows * (cols + pitch) + 16,), 7.0, dtype=x.dtype, device="cuda")
    view = torch.as_strided(buf, (rows, cols), (cols + pitch, 1), shift)
    view.copy_(x.view(rows, cols))
    return view, buf


def untouched_outside(view, buf):
    kept = view.clone()
    view.fill_(7.0)
    ok = bool((buf == 7.0).all())
    view.copy_(kept)
    return ok


def bits(t):
    return t.contiguous().view(torch.uint8)


def pieces(n):
    return [(a, min(a + PIECE, n)) for a in range(0, n, PIECE)]


def in_pieces(tsr, p, g, kind, steps):
    """The same steps, each piece a plan of its own.  Returns the parameter and the moments (the scales last)."""
    p = p.clone()
    out = []
    for a, b in pieces(p.numel()):
        plan = tsr.DensePlan([p[a:b]], [g[a:b]], state_dtype=kind)
        for t in steps:
            plan.step(hyper(tsr, t))
        out.append(plan.states[0])
    return p, [torch.cat([bits(s[k]).view(-1) for s in out]) for k in range(len(out[0]))]


@pytest.mark.parametrize("kind", [torch.float32, F8])
@pytest.mark.parametrize("pd,gd", [("f32", "f32"), ("bf16", "bf16"), ("bf16", "f32"), ("f32", "bf16")])
def test_steps_to_nearest(tsr, pd, gd, kind):
    p0, g0 = rand(N, 1, 0.02).to(DT[pd]), gradient(N, 2).to(DT[gd])
    want, states = in_pieces(tsr, p0, g0, kind, (1, 2))
    for layout in LAYOUTS:
        (p, pbuf), (g, gbuf) = placed(p0, layout), placed(g0, layout)
        image, ibuf = placed(torch.zeros_like(p0, dtype=torch.bfloat16), layout) if pd == "f32" else (None, None)
        plan = tsr.DensePlan([p], [g], state_dtype=kind, images=[image])
        for t in (1, 2):
            plan.step(hyper(tsr, t))
        assert torch.equal(p.reshape(-1), want), layout
        for s, w in zip(plan.states[0], states):
            assert torch.equal(bits(s).view(-1), w), layout
        assert image is None or torch.equal(image, p.bfloat16())
        assert untouched_outside(p, pbuf) and untouched_outside(g, gbuf) and (image is None or untouched_outside(image, ibuf))


@pytest.mark.parametrize("pd,gd", [("f32", "f32"), ("bf16", "bf16"), ("bf16", "f32"), ("f32", "bf16")])
def test_stochastic_8_bit_steps(tsr, pd, gd):
    """Sampled blocks of the first layout against the model's bits; the other layouts against the first."""
    p0, g0 = rand(N, 3, 0.02).to(DT[pd]), gradient(N, 4).to(DT[gd])
    first = None
    for layout in LAYOUTS:
        (p, pbuf), (g, _) = placed(p0, layout), placed(g0, layout)
        plan = tsr.DensePlan([p], [g], state_dtype=F8)
        plan.step(hyper(tsr, 1), rounding=1, seed=11)
        before = [s.clone() for s in plan.states[0]]
        plan.step(hyper(tsr, 2), rounding=1, seed=11)
        assert untouched_outside(p, pbuf)
        if first is None:
            first = [p.reshape(-1)] + list(plan.states[0])
            picked = np.unique(np.concatenate([np.arange(20), np.random.default_rng(1).integers(0, N // BLOCK, 2000), np.arange(N // BLOCK - 20, N // BLOCK)]))
            at = torch.from_numpy(picked).cuda()
            take = lambda x: x.view(torch.uint8)[:N // BLOCK * BLOCK].view(-1, BLOCK)[at].cpu().numpy()  # noqa: E731
            gs = g0.float()[:N // BLOCK * BLOCK].view(-1, BLOCK)[at].cpu().numpy()
            cm, cr, sc = take(before[0]), take(before[1]), before[2][at].cpu().numpy()
            k1, k2 = dm.keys(11, 2, 0)
            F = np.float32
            m = E4M3[cm].astype(F) * sc[:, :1]
            r = E4M3[cr].astype(F) * sc[:, 1:]
            m1 = F(HYPER["beta1"]) * m + F(1.0 - HYPER["beta1"]) * gs
            r1 = np.sqrt(F(HYPER["beta2"]) * (r * r) + F(1.0 - HYPER["beta2"]) * (gs * gs))
            words = dm.random_words((picked[:, None] * BLOCK + np.arange(BLOCK)[None, :]).astype(np.uint32), k1, k2)
            ws = np.concatenate([dm.scale_of(np.abs(m1)), dm.scale_of(r1)], axis=1)
            wm = dm.quantise(m1, ws[:, :1], words & np.uint32(0xFFFF))
            wr = dm.quantise(r1, ws[:, 1:], words >> np.uint32(16))
            wr = np.where((r1 > 0) & (wr == 0), 1, wr)
            assert np.array_equal(plan.states[0][2][at].cpu().numpy(), ws.astype(F))
            assert np.array_equal(E4M3[take(plan.states[0][0])], E4M3[wm])
            assert np.array_equal(take(plan.states[0][1]), wr)
        for a, b in zip(first, [p.reshape(-1)] + list(plan.states[0])):
            assert torch.equal(bits(a), bits(b)), layout


def test_stochastic_parameters_with_fp32_moments_are_the_same_in_every_layout(tsr):
    p0, g0 = rand(N, 5, 0.02).bfloat16(), gradient(N, 6).bfloat16()
    first = None
    for layout in LAYOUTS:
        (p, pbuf), (g, _) = placed(p0, layout), placed(g0, layout)
        plan = tsr.DensePlan([p], [g])
        for t in (1, 2):
            plan.step(hyper(tsr, t), rounding=1, seed=t)
        assert untouched_outside(p, pbuf)
        now = [p.reshape(-1)] + list(plan.states[0])
        first = first or now
        for a, b in zip(first, now):
            assert torch.equal(bits(a), bits(b)), layout


@pytest.mark.parametrize("layout", list(LAYOUTS))
@pytest.mark.parametrize("gd", ["f32", "bf16"])
@pytest.mark.parametrize("rows,cols", [(ROWS, COLS), (300, 100), (4700, 4099), (90_000, 61)])
def test_norm(tsr, gd, rows, cols, layout):
    """Eight squares at a time in FP32 (relative error 9 units), the rest in FP64, one rounding at the end; the root halves the
    relative error."""
    g0 = gradient(rows * cols, 7).to(DT[gd])
    g, _ = placed(g0, layout, rows, cols)
    want = float(g0.double().square().sum().sqrt())
    n, f = tsr.DensePlan(None, [g]).grad_norm(0.3 * want).tolist()
    assert abs(n / want - 1) <= 6 * U24
    assert abs(f - f32(0.3 * want) / (want + 1e-6)) <= 8 * U24


@pytest.mark.parametrize("shift", [0, 1, 2])
def test_conversions(tsr, shift):
    """20 M elements: eight blocks a warp of a conversion's plan.  To 8 bits as small plans do it, to FP32 by value."""
    n = 20_000_077
    def states(kind, off=shift):
        if kind == torch.float32:
            return tuple(torch.full((n + off,), 3.0, device="cuda")[off:] for _ in (0, 1))
        return tuple(torch.full((n + off,), 5, dtype=torch.uint8, device="cuda")[off:].view(F8) for _ in (0, 1)) + (torch.zeros((n + 255) // 256, 2, device="cuda"),)
    m, v = states(torch.float32)
    m.copy_(gradient(n, 8)), v.copy_(gradient(n, 9).square())
    s8, back = states(F8), states(torch.float32)
    a, b, c = (tsr.DensePlan(None, None, states=[s]) for s in ((m, v), s8, back))
    b.copy_state(a)
    c.copy_state(b)
    scale = s8[2].repeat_interleave(BLOCK, 0)[:n]
    assert torch.equal(back[0], s8[0].float() * scale[:, 0])
    assert torch.equal(back[1], (s8[1].float() * scale[:, 1]).square())
    small = states(F8, 0)
    for x, y in pieces(n):
        src = tsr.DensePlan(None, None, states=[(m[x:y], v[x:y])])
        dst = tsr.DensePlan(None, None, states=[(small[0][x:y], small[1][x:y], small[2][x // BLOCK:(y + BLOCK - 1) // BLOCK])])
        dst.copy_state(src)
    for x, y in zip(small, s8):
        assert torch.equal(bits(x), bits(y))
    again, same = states(F8), states(torch.float32)
    tsr.DensePlan(None, None, states=[again]).copy_state(b)
    tsr.DensePlan(None, None, states=[same]).copy_state(a)
    assert all(torch.equal(bits(x), bits(y)) for x, y in zip(again + same, s8 + (m, v)))


def test_a_factor_that_is_not_finite_ends_long_chunks_too(tsr):
    """The ring has loads on their way when the factor is looked at."""
    for kind in (torch.float32, F8):
        for layout in LAYOUTS:
            (p, _), (g, _) = placed(rand(N, 1), layout), placed(rand(N, 2), layout)
            plan = tsr.DensePlan([p], [g], state_dtype=kind)
            plan.step(hyper(tsr, 1))
            before = [x.clone() for x in (p,) + plan.states[0]]
            plan.step(hyper(tsr, 2), grad_scale=torch.tensor([math.nan], device="cuda"), rounding=1, seed=2)
            assert all(torch.equal(bits(x), bits(y)) for x, y in zip(before, (p,) + plan.states[0])), layout

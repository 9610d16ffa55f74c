"""Dense parameters through a plan: AdamW with FP32 and 8-bit states, the gradient norm, state conversion (GPU), against
the definition in 64 bits and, for the 8-bit state, against its bits from IEEE FP32 operations."""
import math

import numpy as np
import pytest
import torch

import dense_model as dm
from dense_model import BLOCK, E4M3, U24, f32, to64

pytestmark = pytest.mark.gpu

F8 = torch.float8_e4m3fn
DT = {"f32": torch.float32, "bf16": torch.bfloat16}
HYPER = dict(lr=f32(2e-3), beta1=f32(0.9), beta2=f32(0.99), eps=f32(1e-8), wd=f32(0.1))


@pytest.fixture(scope="module")
def tsr():
    import paper_2602_08007_b200 as t
    return t


def hyper(tsr, t, **kw):
    h = dict(HYPER, **kw)
    return tsr.make_hyper(t, lr=h["lr"], beta1=h["beta1"], beta2=h["beta2"], eps=h["eps"], weight_decay=h["wd"]), dict(h, t=t)


def rand(shape, seed, scale=1.0):
    gen = torch.Generator().manual_seed(seed)
    return torch.randn(shape, generator=gen) * scale


def gradient(n, seed):
    """Values over many orders of magnitude, with a zero run and a zero block where there is room."""
    g = rand(n, seed) * torch.exp(rand(n, seed + 1) * 2 - 6)
    if n > 600:
        g[256:512] = 0
        g[550:560] = 0
    return g


def place(x, layout, dtype):
    """x (flat) on the GPU: 'plain', 'shifted' (starts one element into an allocation), 'pitched' or 'odd pitch' (as a
    matrix), 'column' (every third element)."""
    x = x.to(dtype)
    n = x.numel()
    if layout == "plain":
        return x.cuda()
    if layout == "shifted":
        buf = torch.zeros(n + 1, dtype=dtype, device="cuda")
        buf[1:].copy_(x)
        return buf[1:]
    if layout == "column":
        buf = torch.zeros(3 * n, dtype=dtype, device="cuda")
        buf[::3].copy_(x)
        return buf[::3]
    cols = next(c for c in ((16, 8, 1) if layout == "pitched" else (7, 5, 3, 1)) if n % c == 0)
    buf = torch.zeros(n // cols, cols + (8 if layout == "pitched" else 2), dtype=dtype, device="cuda")
    buf[:, :cols].copy_(x.view(-1, cols))
    return buf[:, :cols]


def flat64(t):
    return to64(t).reshape(-1)


SIZES = [1, 2, 7, 31, 32, 33, 255, 256, 257, 511, 513, 1000, 4096, 4097, 8191, 70000]


# ---- AdamW, FP32 state ---------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("layout", ["plain", "shifted", "pitched", "odd pitch", "column"])
@pytest.mark.parametrize("pd,gd", [("f32", "f32"), ("f32", "bf16"), ("bf16", "bf16"), ("bf16", "f32")])
def test_step_with_fp32_states(tsr, pd, gd, layout):
    """Three steps over tensors of all sizes at once; each step is compared with the definition from the state it started
    from.  A BF16 parameter is the FP32 result rounded once: half a unit more."""
    ps = [place(rand(n, 10 + n, 0.02), layout, DT[pd]) for n in SIZES]
    gs = [place(gradient(n, 20 + n), layout, DT[gd]) for n in SIZES]
    lm = [1.0 if i % 3 else 0.5 for i in range(len(SIZES))]
    wm = [0.0 if i % 2 else 1.0 for i in range(len(SIZES))]
    plan = tsr.DensePlan(ps, gs, lr_mult=lm, wd_mult=wm)
    clip = torch.tensor([f32(0.37)], device="cuda")
    for t in (1, 2, 3):
        hy, h = hyper(tsr, t)
        for g, n in zip(gs, SIZES):
            g.copy_(gradient(n, 1000 * t + n).to(DT[gd]).view(g.shape))
        before = [(flat64(p), flat64(g), flat64(s[0]), flat64(s[1])) for p, g, s in zip(ps, gs, plan.states)]
        plan.step(hy, grad_scale=clip if t == 2 else None)
        for i, (p, g, m, v) in enumerate(before):
            p1, m1, v1, tp, tm, tv = dm.step64(p, g, m, v, h, f32(0.37) if t == 2 else 1.0, lm[i], wm[i])
            if pd == "bf16":
                tp = tp + 0.5 * dm.bf16_unit(np.abs(p1) + tp)
            for got, want, tol in ((ps[i], p1, tp), (plan.states[i][0], m1, tm), (plan.states[i][1], v1, tv)):
                assert np.all(np.abs(flat64(got) - want) <= tol), (SIZES[i], t)


def test_fp32_states_give_the_bits_of_dense_adamw(tsr):
    ps, gs = [[rand(n, s + n, 0.02).cuda() for n in SIZES] for s in (1, 2)]
    qs = [p.clone() for p in ps]
    ms, vs = [[torch.zeros_like(p) for p in ps] for _ in (0, 1)]
    plan = tsr.DensePlan(ps, gs)
    for t in (1, 2):
        hy, _ = hyper(tsr, t)
        plan.step(hy)
        tsr.dense_adamw(qs, gs, ms, vs, hy)
    for p, q, s, m, v in zip(ps, qs, plan.states, ms, vs):
        assert torch.equal(p, q) and torch.equal(s[0], m) and torch.equal(s[1], v)


def test_padding_between_rows_and_neighbours_in_memory_are_left_alone(tsr):
    """Every element of the buffers that is no element of a tensor keeps its value."""
    for n, cols, ld in ((35 * 50, 35, 40), (64 * 48, 64, 72), (9 * 257, 257, 300)):
        for state in (torch.float32, F8):
            rows = n // cols
            base = torch.full((2 + rows * ld,), 7.0, device="cuda")
            gb = torch.full((rows * ld,), float("nan"), device="cuda")
            img = torch.full((rows * ld,), 5.0, dtype=torch.bfloat16, device="cuda")
            p = torch.as_strided(base, (rows, cols), (ld, 1), 2)
            g = torch.as_strided(gb, (rows, cols), (ld, 1))
            im = torch.as_strided(img, (rows, cols), (ld, 1))
            p.copy_(rand((rows, cols), 5).cuda())
            g.copy_(rand((rows, cols), 6).cuda())
            plan = tsr.DensePlan([p], [g], state_dtype=state, images=[im])
            plan.step(hyper(tsr, 1)[0])
            assert torch.equal(im, p.bfloat16()) and not torch.isnan(p).any()
            mask = torch.ones_like(base, dtype=torch.bool)
            torch.as_strided(mask, (rows, cols), (ld, 1), 2).fill_(False)
            assert (base[mask] == 7.0).all()
            mask = torch.ones_like(img, dtype=torch.bool)
            torch.as_strided(mask, (rows, cols), (ld, 1)).fill_(False)
            assert (img[mask] == 5.0).all()


# ---- AdamW, 8-bit state ----------------------------------------------------------------------------------------------------

def codes(t):
    return t.view(torch.uint8).cpu().numpy().reshape(-1)


def random_state(n, seed):
    """An 8-bit state with every kind of code: both signs, subnormals, zeros."""
    rng = np.random.default_rng(seed)
    nb = (n + BLOCK - 1) // BLOCK
    cm = rng.integers(0, 256, n).astype(np.uint8)
    cm[(cm & 127) == 127] = 0
    cr = rng.integers(0, 127, n).astype(np.uint8)
    scale = 2.0 ** rng.integers(-30, 3, (nb, 2))
    return cm, cr, scale.astype(np.float32)


@pytest.mark.parametrize("layout", ["plain", "shifted", "pitched", "odd pitch", "column"])
@pytest.mark.parametrize("stochastic", [False, True])
@pytest.mark.parametrize("pd,gd", [("f32", "f32"), ("bf16", "bf16"), ("bf16", "f32"), ("f32", "bf16")])
def test_step_with_8_bit_states(tsr, pd, gd, stochastic, layout):
    """Stored bits equal the IEEE model's; the moments they stand for are within one rounding of the definition in 64 bits;
    the parameter is the definition's."""
    ps = [place(rand(n, 10 + n, 0.02), layout, DT[pd]) for n in SIZES]
    gs = [place(gradient(n, 20 + n), layout, DT[gd]) for n in SIZES]
    states = []
    for n in SIZES:
        cm, cr, sc = random_state(n, n)
        states.append((torch.from_numpy(cm).cuda().view(F8), torch.from_numpy(cr).cuda().view(F8), torch.from_numpy(sc).cuda()))
    plan = tsr.DensePlan(ps, gs, states=states)
    clip = torch.tensor([f32(0.37)], device="cuda")
    seed = 0x1234567890ABCDEF
    for t in (7, 8):
        hy, h = hyper(tsr, t)
        s = f32(0.37) if t == 8 else 1.0
        before = [(flat64(p), flat64(g), codes(a), codes(b), c.cpu().numpy().reshape(-1, 2)) for p, g, (a, b, c) in zip(ps, gs, plan.states)]
        plan.step(hy, grad_scale=clip if t == 8 else None, rounding=int(stochastic), seed=seed)
        for i, (p, g, cm, cr, sc) in enumerate(before):
            n = SIZES[i]
            key = dm.keys(seed, t, i) if stochastic else None
            wm, wr, ws, m32, r32 = dm.step_bits(g.astype(np.float32), cm, cr, sc, h, s if t == 8 else None, key)
            gm, gr, gsc = codes(plan.states[i][0]), codes(plan.states[i][1]), plan.states[i][2].cpu().numpy().reshape(-1, 2)
            assert np.array_equal(gsc, ws), (n, t)
            assert np.array_equal(E4M3[gm], E4M3[wm]), (n, t)
            assert np.array_equal(gr, wr), (n, t)
            rep = [np.repeat(sc[:, k].astype(np.float64), BLOCK)[:n] for k in (0, 1)]
            p1, m1, v1, tp, tm, tv = dm.step64(p, g, E4M3[cm] * rep[0], (E4M3[cr] * rep[1]) ** 2, h, s)
            new = [np.repeat(gsc[:, k].astype(np.float64), BLOCK)[:n] for k in (0, 1)]
            part = 1.0 if stochastic else 0.5
            r1 = np.sqrt(v1)
            # FP32 error, then one rounding to E4M3 (a root's floor is one spacing at most)
            assert np.all(np.abs(E4M3[gm] * new[0] - m1) <= 2 * tm + part * dm.spacing(m1 / new[0]) * new[0])
            assert np.all(np.abs(E4M3[gr] * new[1] - r1) <= 8 * U24 * r1 + dm.spacing(r1 / new[1]) * new[1] * (1.0 if stochastic else np.where(r1 / new[1] < 2.0 ** -9, 1.0, 0.5)))
            assert np.all((E4M3[gr] > 0) == (r1 > 0))
            if pd == "bf16":
                tp = tp + (1.0 if stochastic else 0.5) * dm.bf16_unit(np.abs(p1) + tp)
            assert np.all(np.abs(flat64(ps[i]) - p1) <= tp), (n, t)


def test_stochastic_rounding_is_right_in_the_mean(tsr):
    """With g = 0 a step stores beta1 m and sqrt(beta2) r.  Over n equal elements the mean of what is stored has a standard
    deviation of at most half a spacing over sqrt(n); 6 of them are allowed.  The same for BF16 parameters and their decay."""
    n = 1 << 20
    seed = 5
    p = torch.full((n,), 1.2345, dtype=torch.bfloat16, device="cuda")
    start = float(p[0])
    g = torch.zeros(n, dtype=torch.bfloat16, device="cuda")
    m8 = torch.full((n,), 8.5, device="cuda")       # 8, 9, ... are E4M3 values
    m8[::BLOCK] = 448.0                              # holds the block's scale at 1
    r8 = torch.full((n,), 0.011, device="cuda")      # among the subnormals: spacing 2^-9
    r8[::BLOCK] = 448.0
    plan = tsr.DensePlan([p], [g], states=[(m8.to(F8), r8.to(F8), torch.ones(n // BLOCK, 2, device="cuda"))])
    m0, r0 = float(plan.states[0][0][1].float()), float(plan.states[0][1][1].float())
    hy, h = hyper(tsr, 3, beta1=f32(0.97), beta2=f32(0.97), eps=f32(1e30), wd=f32(0.3))   # eps: the update vanishes, decay stays
    plan.step(hy, rounding=tsr.TSR_ROUND_STOCHASTIC, seed=seed)
    keep = torch.ones(n, dtype=torch.bool, device="cuda")
    keep[::BLOCK] = False
    cnt = int(keep.sum())
    scale = plan.states[0][2].double().repeat_interleave(BLOCK, 0)
    for k, want in ((0, h["beta1"] * m0), (1, math.sqrt(h["beta2"]) * r0)):
        x = plan.states[0][k].double() * scale[:, k]
        s = float(scale[1, k])
        step = float(dm.spacing(np.array(want / s))) * s
        assert len(x[keep].unique()) == 2
        assert abs(float(x[keep].mean()) - want) <= 6 * step / 2 / math.sqrt(cnt) + 2.0 ** -16 * step + 8 * U24 * want
    want = start * (1 - h["lr"] * h["wd"])
    step = 2.0 ** -7
    assert len(p.unique()) == 2
    assert abs(float(p.double().mean()) - want) <= 6 * step / 2 / math.sqrt(n) + 2.0 ** -16 * step + 8 * U24


def test_small_changes_accumulate_under_stochastic_rounding_only(tsr):
    """200 steps without gradient at beta2 = 0.999: v decays by 18 %.  To nearest, every root returns to its value at once;
    stochastic, the mean follows."""
    n = 1 << 16
    out = {}
    for rounding in (tsr.TSR_ROUND_NEAREST, tsr.TSR_ROUND_STOCHASTIC):
        p, g = torch.zeros(n, device="cuda"), torch.zeros(n, device="cuda")
        r = torch.exp(rand(n, 3)).cuda()
        r[::BLOCK] = 2.0 ** 6 * 1.75                  # the scale: 2^-2, through the whole run
        states = [(torch.zeros(n, dtype=torch.uint8, device="cuda").view(F8), (r * 4).to(F8), torch.full((n // BLOCK, 2), 0.25, device="cuda"))]
        plan = tsr.DensePlan([p], [g], states=states)
        r0 = plan.states[0][1].double() * 0.25
        for t in range(1, 201):
            plan.step(hyper(tsr, t, beta2=f32(0.999))[0], rounding=rounding, seed=11)
        r1 = plan.states[0][1].double() * plan.states[0][2][:, 1].double().repeat_interleave(BLOCK)
        out[rounding] = float((r1.sum() / r0.sum()).cpu())
    assert out[tsr.TSR_ROUND_NEAREST] == 1.0
    # 200 roundings of relative variance at most (1/16)^2 / 4 ... each, averaged over 65536 independent elements of which the
    # largest (the 256 that fix the scales) carry about half the sum: standard deviation below 0.5 %
    assert abs(out[tsr.TSR_ROUND_STOCHASTIC] - 0.999 ** 100) < 0.02


def test_random_words_depend_on_seed_step_and_tensor_and_nothing_else(tsr):
    def run(seed, t, offset=0, pad=0):
        n = 5000
        ps, gs, st = [], [], []
        for k in range(2 + pad):
            ps.append(torch.zeros(n + offset, device="cuda")[offset:])
            g = torch.zeros(n + offset, device="cuda")[offset:]
            g.copy_(rand(n, 3).cuda())
            gs.append(g)
        plan = tsr.DensePlan(ps, gs, state_dtype=F8)
        plan.step(hyper(tsr, t, beta1=0.0, beta2=0.0)[0], rounding=1, seed=seed)
        return [torch.cat([codes_t.view(torch.uint8) for codes_t in s[:2]]).clone() for s in plan.states]
    a = run(1, 1)
    assert torch.equal(a[0], run(1, 1, offset=3)[0]) and torch.equal(a[1], run(1, 1, pad=3)[1])   # alignment, other tensors
    for other in (a[1], run(2, 1)[0], run(1 << 40 | 1, 1)[0], run(1, 2)[0]):
        differ = float((a[0] != other).float().mean())
        assert 0.1 < differ < 0.9


# ---- values that are not finite, and steps that are not taken --------------------------------------------------------------

@pytest.mark.parametrize("bad", [float("inf"), float("-inf"), float("nan")])
def test_bad_gradients_stay_where_they_are(tsr, bad):
    """FP32 state: that element alone.  8-bit state: the moments of its block of 256, and its own parameter."""
    n, at = 2000, 700
    for rounding in (0, 1):
        res = {}
        for state in (torch.float32, F8):
            for poison in (False, True):
                p, g = rand(n, 1).cuda(), rand(n, 2).cuda()
                if poison:
                    g[at] = bad
                plan = tsr.DensePlan([p], [g], state_dtype=state)
                plan.step(hyper(tsr, 1)[0], rounding=rounding, seed=3)
                s = plan.states[0]
                mv = s if state == torch.float32 else tuple(s[k].float() * s[2][:, k].repeat_interleave(BLOCK)[:n] for k in (0, 1))
                res[state, poison] = (p,) + tuple(mv)
        others = torch.arange(n, device="cuda") != at
        block = torch.arange(n, device="cuda") // BLOCK == at // BLOCK
        for k in range(3):
            clean, bad_ = res[torch.float32, False][k], res[torch.float32, True][k]
            assert torch.equal(clean[others], bad_[others])
        assert not torch.isfinite(res[torch.float32, True][0][at])
        clean, bad_ = res[F8, False], res[F8, True]
        assert torch.equal(clean[0][others], bad_[0][others]) and not torch.isfinite(bad_[0][at])
        for k in (1, 2):
            assert torch.equal(clean[k][~block], bad_[k][~block]) and torch.isnan(bad_[k][block]).all()


@pytest.mark.parametrize("state", [torch.float32, F8])
def test_step_with_a_factor_that_is_not_finite_changes_nothing(tsr, state):
    p, g = rand(3000, 1).cuda(), rand(3000, 2).cuda()
    im = torch.zeros_like(p, dtype=torch.bfloat16)
    plan = tsr.DensePlan([p], [g], state_dtype=state, images=[im])
    plan.step(hyper(tsr, 1)[0])
    before = [x.clone() for x in (p, im) + plan.states[0]]
    for f in (float("nan"), float("inf"), float("-inf")):
        plan.step(hyper(tsr, 2)[0], grad_scale=torch.tensor([f], device="cuda"))
        assert all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip(before, (p, im) + plan.states[0]))
    plan.step(hyper(tsr, 2)[0], grad_scale=torch.tensor([0.0], device="cuda"))
    assert not torch.equal(before[0], p)


@pytest.mark.parametrize("state", [torch.float32, F8])
def test_extreme_values(tsr, state):
    """Zero gradients on zero states change nothing but the decay; tiny and huge ones give finite results where FP32 has
    them; elements far below their block's largest take steps no larger than theirs."""
    n = 1024
    p, g = rand(n, 1).cuda(), torch.zeros(n, device="cuda")
    p0 = p.clone()
    plan = tsr.DensePlan([p], [g], state_dtype=state, wd_mult=[0.0])
    plan.step(hyper(tsr, 1)[0])
    assert torch.equal(p, p0)
    g[:256] = 1e-30
    g[256:512] = 1e15 * torch.where(torch.arange(256, device="cuda") % 2 == 0, 1.0, -1.0)
    g[512:768] = torch.logspace(-30, 3, 256, device="cuda")
    plan.step(hyper(tsr, 2)[0])
    assert torch.isfinite(p).all()
    for t in range(3, 30):       # no gradient from here: sums of m / sqrt(v) stay bounded, roots do not vanish before m
        g.zero_()
        plan.step(hyper(tsr, t)[0])
        assert torch.isfinite(p).all()
        # |m_hat| / sqrt(v_hat) after one gradient: (1-b1) b1^k / sqrt((1-b2) b2^k) times the bias corrections, at most 10
        # times lr a step in FP32; an 8-bit root is at most one spacing too small
        assert float((p - p0).abs().max()) <= t * 12 * HYPER["lr"]


# ---- plans -------------------------------------------------------------------------------------------------------------------

def test_mixed_types_in_one_plan_equal_single_plans(tsr):
    kinds = [(pd, gd, st) for pd in DT for gd in DT for st in (torch.float32, F8)] * 2
    def make():
        return ([place(rand(300 + 37 * i, i), "plain", DT[k[0]]) for i, k in enumerate(kinds)],
                [place(rand(300 + 37 * i, 50 + i), "plain", DT[k[1]]) for i, k in enumerate(kinds)])
    ps, gs = make()
    plan = tsr.DensePlan(ps, gs, state_dtype=[k[2] for k in kinds])
    qs, hs = make()
    plan.step(hyper(tsr, 1)[0])
    for i, k in enumerate(kinds):
        one = tsr.DensePlan([qs[i]], [hs[i]], state_dtype=k[2])
        one.step(hyper(tsr, 1)[0])
        assert torch.equal(ps[i], qs[i])
        for a, b in zip(plan.states[i], one.states[0]):
            assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))


def test_empty_plans_and_empty_tensors(tsr):
    plan = tsr.DensePlan([], [])
    plan.step(hyper(tsr, 1)[0])
    assert plan.grad_norm(1.0).tolist() == [0.0, 1.0]
    plan.copy_state(tsr.DensePlan([], []))
    p = [torch.zeros(0, device="cuda"), torch.ones(3, device="cuda"), torch.zeros(4, 0, device="cuda")]
    g = [torch.zeros(0, device="cuda"), torch.full((3,), 2.0, device="cuda"), torch.zeros(4, 0, device="cuda")]
    for state in (torch.float32, F8):
        plan = tsr.DensePlan(p, g, state_dtype=state)
        plan.step(hyper(tsr, 1)[0])
        assert abs(float(plan.grad_norm(1.0)[0]) - math.sqrt(12)) < 1e-5


def test_many_tensors(tsr):
    """More tensors than any table in kernel parameters could hold."""
    k = 3000
    flat_p, flat_g = torch.zeros(k * 5, device="cuda"), rand(k * 5, 1).cuda()
    ps, gs = list(flat_p.split(5)), list(flat_g.split(5))
    plan = tsr.DensePlan(ps, gs)
    plan.step(hyper(tsr, 1, wd=0.0)[0])
    assert torch.allclose(flat_p, -HYPER["lr"] * flat_g / (flat_g.abs() + HYPER["eps"]), rtol=1e-4)
    assert abs(float(plan.grad_norm()[0]) / float(flat_g.double().norm()) - 1) < 1e-6


def test_offsets_beyond_32_bits(tsr):
    """A tensor of more than 2^31 elements: its ends are compared with small tensors of the same values."""
    n = (1 << 31) + 12345
    if torch.cuda.mem_get_info()[0] < 40 << 30:
        pytest.skip("needs 40 GB of free device memory")
    p = torch.zeros(n, dtype=torch.bfloat16, device="cuda")
    g = torch.zeros(n, dtype=torch.bfloat16, device="cuda")
    k = n - n // BLOCK * BLOCK + 10 * BLOCK       # the last blocks, the partial one among them
    g[:k] = rand(k, 1).cuda().bfloat16()
    g[-k:] = rand(k, 2).cuda().bfloat16()
    plan = tsr.DensePlan([p], [g], state_dtype=F8)
    plan.step(hyper(tsr, 1)[0])
    for part, seed in ((slice(None, k), 1), (slice(n - k, None), 2)):
        q, h = torch.zeros(k, dtype=torch.bfloat16, device="cuda"), rand(k, seed).cuda().bfloat16()
        one = tsr.DensePlan([q], [h], state_dtype=F8)
        one.step(hyper(tsr, 1)[0])
        assert torch.equal(p[part], q)
        for a, b in ((plan.states[0][0][part], one.states[0][0]), (plan.states[0][1][part], one.states[0][1])):
            assert torch.equal(a.view(torch.uint8)[:k // BLOCK * BLOCK], b.view(torch.uint8)[:k // BLOCK * BLOCK])
    want = math.sqrt(float((g[:k].double() ** 2).sum() + (g[-k:].double() ** 2).sum()))
    assert abs(float(plan.grad_norm()[0]) / want - 1) < 2e-7
    back = tsr.DensePlan(None, None, states=[(torch.zeros(n, device="cuda"), torch.zeros(n, device="cuda"))])
    back.copy_state(plan)
    s = plan.states[0]
    assert torch.equal(back.states[0][0][-BLOCK:], (s[0].view(torch.uint8)[-BLOCK:].view(F8).float() * s[2][(n - BLOCK) // BLOCK:, 0].repeat_interleave(BLOCK)[(n - BLOCK) % BLOCK:][:BLOCK]))


@pytest.mark.parametrize("shift", [0, 1])
def test_random_words_beyond_32_bits(tsr, shift):
    """More than 2^32 elements: the words of a BF16 parameter count pairs, modulo 2^32 pairs, those of the state elements,
    modulo 2^32 elements, on both sides of the 32-bit border."""
    n = (1 << 32) + 8192
    if torch.cuda.mem_get_info()[0] < 40 << 30:
        pytest.skip("needs 40 GB of free device memory")
    p = torch.full((n + shift,), 1.2345, dtype=torch.bfloat16, device="cuda")[shift:]
    g = torch.zeros(n + shift, dtype=torch.bfloat16, device="cuda")[shift:]
    zero = lambda: torch.zeros(n, dtype=torch.uint8, device="cuda")  # noqa: E731
    m8 = zero()
    m8 += 0x51                                                         # the E4M3 value 9
    plan = tsr.DensePlan([p], [g], states=[(m8.view(F8), zero().view(F8), torch.ones((n + BLOCK - 1) // BLOCK, 2, device="cuda"))])
    start = np.float32(p[0].item())
    seed, t = 77, 5
    hy, h = hyper(tsr, t, eps=f32(1e30), wd=f32(0.3))
    plan.step(hy, rounding=tsr.TSR_ROUND_STOCHASTIC, seed=seed)
    k1, k2 = dm.keys(seed, t, 0)
    F = np.float32
    decayed = start * (F(1) - F(h["lr"]) * F(h["wd"]))
    m1 = F(h["beta1"]) * F(9)
    for at in (0, (1 << 32) - 4096, 1 << 32, n - 4096):
        e = np.arange(at, at + 4096, dtype=np.uint64)
        w = dm.random_words((e >> 1).astype(np.uint32), k1 ^ 0x5BD1E995, k2)
        u = np.where(e & 1, w >> 16, w & 0xFFFF).astype(np.uint32)
        want = ((decayed.view(np.uint32) + u) & np.uint32(0xFFFF0000)).view(np.float32)
        assert np.array_equal(p[at:at + 4096].float().cpu().numpy(), want)
        w = dm.random_words(e.astype(np.uint32), k1, k2)
        scale = dm.scale_of(np.full((1, 1), m1))
        code = dm.quantise(np.full(4096, m1, F), scale[0, 0], w & np.uint32(0xFFFF))
        assert np.array_equal(codes(plan.states[0][0][at:at + 4096]), code)


@pytest.mark.parametrize("cols,ld", [(5461, 5464), (1, 3), (31, 33)])
def test_pitched_matrices_step_like_contiguous_ones(tsr, cols, ld):
    rows = 37
    a = torch.zeros(rows, ld, device="cuda")[:, :cols]
    b = torch.zeros(rows, ld + 5, dtype=torch.bfloat16, device="cuda")[:, :cols]
    a.copy_(rand((rows, cols), 1).cuda())
    b.copy_(rand((rows, cols), 2).cuda())
    p, g = a.contiguous(), b.contiguous()
    for x, y in ((a, b), (a.clone(), g)):       # both pitched; (a contiguous copy) and its dense gradient
        x2, ref_p = x, p.clone()
        for state in (torch.float32, F8):
            start = x2.clone()
            q = p.clone()
            x2.copy_(p)
            plan, one = tsr.DensePlan([x2], [y], state_dtype=state), tsr.DensePlan([q], [g], state_dtype=state)
            plan.step(hyper(tsr, 1)[0], rounding=1, seed=9)
            one.step(hyper(tsr, 1)[0], rounding=1, seed=9)
            assert torch.equal(x2, q)
            assert abs(float(plan.grad_norm()[0]) / float(one.grad_norm()[0]) - 1) <= 12 * U24    # another order of summation
            for u, w in zip(plan.states[0], one.states[0]):
                assert torch.equal(u.view(torch.uint8), w.view(torch.uint8))


@pytest.mark.parametrize("stochastic", [0, 1])
@pytest.mark.parametrize("state", [torch.float32, F8])
@pytest.mark.parametrize("pd,gd", [("f32", "f32"), ("bf16", "bf16"), ("bf16", "f32"), ("f32", "bf16")])
def test_every_alignment_gives_the_same_bits(tsr, pd, gd, state, stochastic):
    """Parameters, gradients and images at all distances from a 16-byte border, contiguous and with rows of many lengths,
    against aligned contiguous copies; what lies before and behind a tensor and between its rows stays as it is."""
    shapes = [(1, 3 * 2048 + 300), (9, 1000), (40, 257), (5, 256), (3, 4099), (30, 100)]
    for rows, cols in shapes:
        n = rows * cols
        p0, g0 = rand((rows, cols), cols, 0.02).to(DT[pd]).cuda(), gradient(n, cols).view(rows, cols).to(DT[gd]).cuda()
        ref = p0.clone()
        image0 = torch.zeros(rows, cols, dtype=torch.bfloat16, device="cuda") if pd == "f32" else None
        one = tsr.DensePlan([ref], [g0], state_dtype=state, images=[image0])
        for t in (1, 2):
            one.step(hyper(tsr, t)[0], rounding=stochastic, seed=t)
        norm = float(one.grad_norm()[0])
        for shift in range(9):
            pitches = [cols] if rows == 1 else [cols, cols + 1 + shift % 5, cols + 3]
            bufs, views = [], []
            for k, (x, extra) in enumerate(((p0, 0), (g0, 1)) + (((image0, 2),) if image0 is not None else ())):
                ld = pitches[(shift + k) % len(pitches)]
                at = (shift * (k + 1) + k) % 9
                buf = torch.full((at + rows * ld + 16,), 7.0, dtype=x.dtype, device="cuda")
                view = torch.as_strided(buf, (rows, cols), (ld, 1), at)
                view.copy_(x)
                bufs.append(buf)
                views.append(view)
            plan = tsr.DensePlan([views[0]], [views[1]], state_dtype=state, images=[views[2]] if image0 is not None else None)
            for t in (1, 2):
                plan.step(hyper(tsr, t)[0], rounding=stochastic, seed=t)
            assert torch.equal(views[0], ref) and (image0 is None or torch.equal(views[2], image0)), (rows, cols, shift)
            assert torch.equal(views[1], g0)
            for a, b in zip(plan.states[0], one.states[0]):
                assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))
            for buf, view in zip(bufs, views):
                view.fill_(7.0)
                assert (buf == 7.0).all()
                view.copy_(g0 if view is views[1] else ref)
            assert abs(float(plan.grad_norm()[0]) / norm - 1) <= 12 * U24


def test_steps_are_ordered_on_their_stream_and_repeat_bit_for_bit(tsr):
    """norm -> step chains on a side stream, behind and before torch kernels, against the default stream."""
    def chain(stream):
        with torch.cuda.stream(stream):
            p, g = rand(300_000, 1).cuda(), torch.zeros(300_000, device="cuda")
            src = rand(300_000, 2).cuda()
            plan = tsr.DensePlan([p], [g], state_dtype=F8)
            for t in range(1, 20):
                g.copy_(src * t)
                f = plan.grad_norm(5.0)
                plan.step(hyper(tsr, t)[0], grad_scale=f[1:], rounding=1, seed=t)
                src += p
            stream.synchronize()
        return p, plan.states[0]
    p1, s1 = chain(torch.cuda.current_stream())
    p2, s2 = chain(torch.cuda.Stream())
    assert torch.equal(p1, p2) and all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip(s1, s2))


def test_a_step_can_be_captured_in_a_graph(tsr):
    p, g = rand(5000, 1).cuda(), rand(5000, 2).cuda()
    q = p.clone()
    a, b = tsr.DensePlan([p], [g]), tsr.DensePlan([q], [g])
    hy, _ = hyper(tsr, 4)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        f = a.grad_norm(0.5)
        a.step(hy, grad_scale=f[1:])
    for _ in range(3):
        graph.replay()
        b.step(hy, grad_scale=b.grad_norm(0.5)[1:])
    assert torch.equal(p, q)


def test_rebinding_follows_the_lists(tsr):
    p, g = torch.zeros(100, device="cuda"), torch.ones(100, device="cuda")
    plan = tsr.DensePlan([p], [g])
    plan.step(hyper(tsr, 1)[0])
    plan.grads[0] = -torch.ones(100, device="cuda")
    plan.bind()
    assert plan.states[0][0].abs().max() > 0        # states stay
    plan.step(hyper(tsr, 2)[0])
    assert float(plan.states[0][0].abs().max()) < 0.011


# ---- norm ----------------------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("layout", ["plain", "shifted", "pitched", "odd pitch", "column"])
@pytest.mark.parametrize("gd", ["f32", "bf16"])
def test_grad_norm(tsr, gd, layout):
    """Sums of eight squares in FP32 (relative error 9 units), the rest in FP64, one rounding at the end; the root halves
    the relative error."""
    gs = [place(gradient(n, n), layout, DT[gd]) for n in SIZES]
    plan = tsr.DensePlan(None, gs)
    want = math.sqrt(sum(float((flat64(g) ** 2).sum()) for g in gs))
    for max_norm in (0.5 * want, 2 * want, math.inf):
        n, f = plan.grad_norm(max_norm).tolist()
        assert abs(n / want - 1) <= 6 * U24
        assert abs(f - min(1.0, f32(max_norm) / (want + 1e-6))) <= 8 * U24
    with_params = tsr.DensePlan([g.float() for g in gs], gs, norm_only=gs)      # every gradient twice
    assert abs(float(with_params.grad_norm()[0]) / (want * math.sqrt(2)) - 1) <= 6 * U24


@pytest.mark.parametrize("value", [1e-30, 1e-22, 1e18, 1e25, 1e37])
def test_norm_of_squares_outside_fp32(tsr, value):
    g = torch.zeros(5000, device="cuda")
    g[7::100] = value
    want = math.sqrt(50) * f32(value)
    out = tsr.DensePlan(None, [g]).grad_norm(1.0)
    assert abs(float(out[0]) / want - 1) <= 6 * U24
    assert abs(float(out[1]) / min(1.0, 1.0 / (want + 1e-6)) - 1) <= 6 * U24
    g[13] = 1.0                                      # the large and the small in one sum
    assert abs(float(tsr.DensePlan(None, [g]).grad_norm()[0]) / math.hypot(want, 1.0) - 1) <= 6 * U24


@pytest.mark.parametrize("value", [math.inf, -math.inf, math.nan, 3e38])
def test_norm_that_is_not_finite_gives_a_factor_that_skips(tsr, value):
    g = rand(10_000, 1).cuda()
    g[4321] = value
    g[4322] = value
    n, f = tsr.DensePlan(None, [g]).grad_norm(1.0).tolist()
    assert not math.isfinite(n) and math.isnan(f)


# ---- conversion ------------------------------------------------------------------------------------------------------------------

def moments(n, seed):
    m = gradient(n, seed)
    v = gradient(n, seed + 7) ** 2
    return m.cuda(), v.cuda()


@pytest.mark.parametrize("shift", [0, 1])
def test_states_convert_both_ways(tsr, shift):
    """FP32 to 8 bits is the stored form's definition bit for bit, 8 bits to FP32 exact, and a second conversion to 8 bits
    keeps every value (a block whose largest value was rounded down to 224 S may go on with S / 2)."""
    f32s, f8s = [], []
    for n in SIZES:
        m, v = moments(n, n)
        f32s.append(tuple(torch.cat([torch.zeros(shift, device="cuda"), x])[shift:] for x in (m, v)))
        f8s.append(tuple(torch.zeros(n + shift, dtype=torch.uint8, device="cuda")[shift:].view(F8) for _ in (0, 1)) +
                   (torch.full(((n + BLOCK - 1) // BLOCK, 2), 9.0, device="cuda"),))
    a, b = tsr.DensePlan(None, None, states=f32s), tsr.DensePlan(None, None, states=f8s)
    b.copy_state(a)
    for (m, v), (cm, cr, sc), n in zip(f32s, f8s, SIZES):
        m, r = m.cpu().numpy(), np.sqrt(v.cpu().numpy())
        bm, br = dm.blocks(m), dm.blocks(r)
        want = np.concatenate([dm.scale_of(np.abs(bm)), dm.scale_of(br)], axis=1)
        assert np.array_equal(sc.cpu().numpy(), want)
        wr = dm.quantise(br, want[:, 1:])
        assert np.array_equal(E4M3[codes(cm)], E4M3[dm.quantise(bm, want[:, :1]).reshape(-1)[:n]])
        assert np.array_equal(codes(cr), np.where((br > 0) & (wr == 0), 1, wr).reshape(-1)[:n])
    back = [tuple(torch.full((n,), 3.0, device="cuda") for _ in (0, 1)) for n in SIZES]
    c = tsr.DensePlan(None, None, states=back)
    c.copy_state(b)
    for (m, v), (cm, cr, sc), n in zip(back, f8s, SIZES):
        s = [np.repeat(sc.cpu().numpy()[:, k].astype(np.float64), BLOCK)[:n] for k in (0, 1)]
        assert np.array_equal(to64(m), E4M3[codes(cm)] * s[0])
        r = E4M3[codes(cr)] * s[1]
        assert np.all(np.abs(to64(v) - r * r) <= U24 * r * r + 2.0 ** -149)
    again = [tuple(torch.zeros(n, dtype=torch.uint8, device="cuda").view(F8) for _ in (0, 1)) + (torch.zeros((n + 255) // 256, 2, device="cuda"),) for n in SIZES]
    d = tsr.DensePlan(None, None, states=again)
    d.copy_state(c)
    e = tsr.DensePlan(None, None, states=[tuple(torch.zeros_like(x) for x in s) for s in back])
    e.copy_state(c)
    for x, y, z, w in zip(again, f8s, e.states, back):
        for k in (0, 1):
            a1, b1 = (s[k].float() * s[2][:, k].repeat_interleave(BLOCK)[:s[k].numel()] for s in (x, y))
            assert torch.equal(a1, b1)
        assert all(torch.equal(i, j) for i, j in zip(z, w))


@pytest.mark.parametrize("shift", [0, 1, 2])
def test_equal_forms_are_copied_as_they_are(tsr, shift):
    """All 256 codes, NaN among them, NaN scales, and FP32 moments with NaN and infinities: byte for byte."""
    for n in (1, 255, 1000, 5000):
        def codes_of(k):
            return (torch.arange(n + shift, device="cuda") * k).to(torch.uint8)[shift:].view(F8)
        scale = torch.full(((n + 255) // 256, 2), 0.5, device="cuda")
        scale[-1, 1] = math.nan
        zeros = lambda: torch.zeros(n + 1, dtype=torch.uint8, device="cuda")[1:].view(F8)  # noqa: E731
        a, b = tsr.DensePlan(None, None, states=[(codes_of(1), codes_of(7), scale)]), tsr.DensePlan(None, None, states=[(zeros(), zeros(), torch.zeros_like(scale))])
        b.copy_state(a)
        assert all(torch.equal(x.view(torch.uint8), y.view(torch.uint8)) for x, y in zip(a.states[0], b.states[0]))
        m, v = (rand(n + shift, k).cuda()[shift:] for k in (1, 2))
        m[0], v[n // 2], v[-1] = math.nan, math.inf, -math.inf
        a, b = (tsr.DensePlan(None, None, states=[s]) for s in ((m, v), (torch.zeros(n, device="cuda"), torch.zeros(n, device="cuda"))))
        b.copy_state(a)
        assert all(torch.equal(x.contiguous().view(torch.int32), y.contiguous().view(torch.int32)) for x, y in zip(a.states[0], b.states[0]))


def test_conversion_between_plans_that_step(tsr):
    """A run with FP32 states goes on with 8-bit ones: the first step afterwards starts from the converted moments."""
    ps, gs = [rand(n, n).cuda() for n in SIZES], [gradient(n, n).cuda() for n in SIZES]
    a = tsr.DensePlan(ps, gs)
    a.step(hyper(tsr, 1)[0])
    b = tsr.DensePlan(ps, gs, state_dtype=F8, norm_only=[gs[0]])
    with pytest.raises(tsr.TsrError) as ei:
        b.copy_state(a)                              # one plan lists a tensor more
    assert ei.value.status == 2
    b = tsr.DensePlan(ps, gs, state_dtype=F8)
    b.copy_state(a)
    qs = [p.clone() for p in ps]
    c = tsr.DensePlan(qs, gs)
    c.copy_state(b)
    b.step(hyper(tsr, 2)[0])
    c.step(hyper(tsr, 2)[0])
    for p, q in zip(ps, qs):                         # the same moments: quotients within their rounding
        assert float((p - q).abs().max()) <= 64 * U24 * (float(q.abs().max()) + HYPER["lr"])


# ---- refusals ----------------------------------------------------------------------------------------------------------------------

def test_refusals(tsr):
    x = torch.zeros(8, 8, device="cuda")
    v = torch.zeros(64, device="cuda")
    f8 = torch.zeros(64, dtype=torch.uint8, device="cuda").view(F8)
    for args, kw in [
        (([x], []), {}), (([x], [x.half()]), {}), (([x.double()], [x]), {}), (([x], [x[:4]]), {}), (([x.t()], [x.t()]), {}),
        (([x.expand(3, 8, 8)], [x.expand(3, 8, 8)]), {}), (([v[:1].expand(64)], [v]), {}), (([x], [x.cpu()]), {}), (([x.cpu()], [x.cpu()]), {}),
        (([x], [x]), dict(images=[x])), (([x], [x]), dict(state_dtype=torch.float16)), (([x], [x]), dict(lr_mult=[1.0, 2.0])),
        (([x], [x]), dict(states=[(v,)])), (([x], [x]), dict(states=[(v, f8)])), (([x], [x]), dict(states=[(v[:63], v)])),
        (([x], [x]), dict(states=[(f8, f8, torch.zeros(1, device="cuda"))])), (([x], [x]), dict(states=[])), ((None, [x]), dict(states=[(v, v)])),
    ]:
        with pytest.raises(ValueError):
            tsr.DensePlan(*args, **kw)
    with pytest.raises(tsr.TsrError) as ei:          # a BF16 parameter has no image
        tsr.DensePlan([x.bfloat16()], [x], images=[x.bfloat16()])
    assert ei.value.status == 1
    with pytest.raises(tsr.TsrError):
        tsr.DensePlan([x], [x], lr_mult=[float("nan")])
    plan = tsr.DensePlan([x], [x.clone()])
    for call, status in [
        (lambda: plan.step(tsr.make_hyper(0)), 1), (lambda: plan.step(tsr.make_hyper(1, rule=tsr.TSR_RULE_SGD)), 1),
        (lambda: plan.step(tsr.make_hyper(1, beta1=1.0)), 1), (lambda: plan.step(tsr.make_hyper(1, beta2=-0.1)), 1),
        (lambda: plan.step(tsr.make_hyper(1), rounding=2), 1), (lambda: plan.grad_norm(0.0), 1), (lambda: plan.grad_norm(-1.0), 1),
        (lambda: plan.grad_norm(float("nan")), 1), (lambda: plan.copy_state(tsr.DensePlan([v[:5]], [v[:5]])), 2),
    ]:
        with pytest.raises(tsr.TsrError) as ei:
            call()
        assert ei.value.status == status
    for bad in (torch.ones(1), torch.ones(1, device="cuda", dtype=torch.float64), torch.ones(0, device="cuda")):
        with pytest.raises(ValueError):
            plan.step(tsr.make_hyper(1), grad_scale=bad)
        with pytest.raises(ValueError):
            plan.grad_norm(1.0, out=bad)
    assert not x.any()


def test_the_example_trains(tsr):
    """TSR blocks and dense parameters under one clipping factor: from the loss of a uniform guess, ln 512, towards the
    entropy of the synthetic text, 0.91."""
    import importlib.util
    import os
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "pretrain_small.py")
    spec = importlib.util.spec_from_file_location("pretrain_small", path)
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    losses, norms = example.train(steps=80)
    assert abs(losses[0] - math.log(512)) < 0.1
    assert all(math.isfinite(x) for x in losses + norms)
    assert sum(losses[-5:]) / 5 < losses[0] - 1.0

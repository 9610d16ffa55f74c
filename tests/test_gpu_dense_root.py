"""The root that the 8-bit state holds, where squares are small: its codes against IEEE FP32 operations (GPU)."""
import numpy as np
import pytest
import torch

import dense_model as dm
from dense_model import BLOCK, f32

pytestmark = pytest.mark.gpu

F8 = torch.float8_e4m3fn
H = dict(lr=f32(2e-3), beta1=f32(0.9), beta2=f32(0.99), eps=f32(1e-8), wd=f32(0.1), t=1)


@pytest.fixture(scope="module")
def tsr():
    import paper_2602_08007_b200 as t
    return t


def codes(t):
    return t.view(torch.uint8).cpu().numpy().reshape(-1)


def model(g, rkeys):
    """Codes and scales after one step from a zero state: the moments' terms are rounded to FP32 and count as zero below
    2^-126, where the state's definition ends."""
    F = np.float32
    omb1, omb2 = F(1.0 - H["beta1"]), F(1.0 - H["beta2"])
    with np.errstate(under="ignore"):
        m, v = omb1 * g, omb2 * (g * g)
    m, v = (np.where(np.abs(x) < F(2.0 ** -126), F(0), x) for x in (m, v))
    bm, br = dm.blocks(m), dm.blocks(np.sqrt(v))
    scale = np.concatenate([dm.scale_of(np.abs(bm)), dm.scale_of(br)], axis=1)
    bits = (None, None)
    if rkeys is not None:
        w = dm.random_words(np.arange(bm.size, dtype=np.uint32), *rkeys).reshape(bm.shape)
        bits = (w & np.uint32(0xFFFF), w >> np.uint32(16))
    cm, cr = dm.quantise(bm, scale[:, :1], bits[0]), dm.quantise(br, scale[:, 1:], bits[1])
    return cm.reshape(-1), np.where((br > 0) & (cr == 0), 1, cr).astype(np.uint8).reshape(-1), scale.astype(F)


def check(tsr, g, shift, rounding):
    """One step from a zero state, codes and scales against the model; g: float32, whole blocks."""
    n = len(g)
    buf = torch.zeros(n + shift, device="cuda")
    x = buf[shift:]
    x.copy_(torch.from_numpy(g).cuda())
    p = torch.zeros(n + shift, device="cuda")[shift:]
    plan = tsr.DensePlan([p], [x], state_dtype=F8)
    plan.step(tsr.make_hyper(1, lr=H["lr"], beta1=H["beta1"], beta2=H["beta2"], eps=H["eps"], weight_decay=H["wd"]), rounding=rounding, seed=5)
    wm, wr, ws = model(g, dm.keys(5, 1, 0) if rounding else None)
    m8, r8, scale = plan.states[0]
    assert np.array_equal(scale.cpu().numpy(), ws)
    assert np.array_equal(codes(r8), wr)
    assert np.array_equal(dm.E4M3[codes(m8)], dm.E4M3[wm])


def squares_near_ties():
    """Gradients whose new v lies within a few units of the square of a number half-way between two E4M3 values, for v from
    2^-126 on: where a root that is off by its last bit gets another code.  Each block holds one much larger root."""
    F = np.float32
    omb2 = 1.0 - H["beta2"]
    out = []
    for k in range(-63, -49):
        near = []
        for i in range(8):
            g = F(np.sqrt(((1 + (2 * i + 1) / 16.0) * 2.0 ** k) ** 2 / omb2))
            near.append((g.view(np.uint32) + np.arange(-42, 43, dtype=np.int64)).astype(np.uint32).view(F))
        near = np.concatenate(near)
        v = F(omb2) * (near * near)
        near = near[v >= F(2.0 ** -126)]
        near = near[:len(near) // (BLOCK - 1) * (BLOCK - 1)].reshape(-1, BLOCK - 1)
        out.append(np.concatenate([near, np.full((len(near), 1), 2.0 ** (k + 6), F)], axis=1).reshape(-1))
    return np.concatenate(out).astype(F)


@pytest.mark.parametrize("rounding", [0, 1])
@pytest.mark.parametrize("shift", [0, 1])
def test_roots_of_small_squares_near_ties(tsr, shift, rounding):
    check(tsr, squares_near_ties(), shift, rounding)


@pytest.mark.parametrize("rounding", [0, 1])
@pytest.mark.parametrize("shift", [0, 1])
def test_roots_over_the_whole_range(tsr, shift, rounding):
    """v from below 2^-126, where it counts as zero, to 2^60; blocks of one size, and blocks that hold all of them."""
    rng = np.random.default_rng(3)
    size = np.repeat(rng.uniform(-66, 32, 400), BLOCK)
    size[:100 * BLOCK] = rng.uniform(-66, 32, 100 * BLOCK)
    g = rng.standard_normal(len(size)) * 2.0 ** size
    g[rng.integers(0, len(g), 2000)] = 0
    check(tsr, g.astype(np.float32), shift, rounding)

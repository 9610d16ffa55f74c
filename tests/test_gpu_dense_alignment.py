"""Dense plans whose moments lie off the alignment that vectors want: the bits are those of aligned moments, and nothing beside
the tensors and the workspace is written (GPU)."""
import ctypes

import pytest
import torch

pytestmark = pytest.mark.gpu

F8 = torch.float8_e4m3fn
GUARD = 64


@pytest.fixture(scope="module")
def tsr():
    import paper_2602_08007_b200 as t
    return t


def rand(shape, seed, scale=1.0):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn(shape, generator=gen, device="cuda") * scale


def bits(t):
    return t.contiguous().view(torch.uint8)


def moment(n, kind, off):
    """A zero moment that starts `off` elements into a buffer of guards, and the buffer."""
    if kind == torch.float32:
        buf = torch.full((off + n + GUARD,), 7.0, device="cuda")
    else:
        buf = torch.full((off + n + GUARD,), 77, dtype=torch.uint8, device="cuda")
    x = buf[off:off + n]
    x.zero_()
    return (x if kind == torch.float32 else x.view(kind)), buf


def guards_left(buf, off, n):
    value = 7.0 if buf.dtype == torch.float32 else 77
    return bool((buf[:off] == value).all()) and bool((buf[off + n:] == value).all())


def state(n, kind, off_m, off_v):
    m, buf_m = moment(n, kind, off_m)
    v, buf_v = moment(n, kind, off_v)
    scale = () if kind == torch.float32 else (torch.zeros((n + 255) // 256, 2, device="cuda"),)
    return (m, v) + scale, lambda: guards_left(buf_m, off_m, n) and guards_left(buf_v, off_v, n)


def matrix(x, pitch):
    rows, cols = x.shape
    buf = torch.zeros(rows, cols + pitch, dtype=x.dtype, device="cuda")
    buf[:, :cols].copy_(x)
    return buf[:, :cols]


def compare(tsr, rows, cols, kind, pd, gd, offsets, pitch, rounding):
    """Two steps with moments `offsets` elements off, against aligned moments of contiguous tensors."""
    n = rows * cols
    p0 = rand((rows, cols), 1, 0.02).to(pd)
    g0 = (rand((rows, cols), 2) * torch.exp(2 * rand((rows, cols), 3) - 6)).to(gd)
    ref = p0.clone()
    one = tsr.DensePlan([ref], [g0], state_dtype=kind)
    hyper = lambda t: tsr.make_hyper(t, lr=2e-3, beta2=0.99, weight_decay=0.1)  # noqa: E731
    for t in (1, 2):
        one.step(hyper(t), rounding=rounding, seed=t)
    p, g = matrix(p0, pitch), matrix(g0, pitch)
    st, guards = state(n, kind, *offsets)
    plan = tsr.DensePlan([p], [g], states=[st])
    # a workspace of exactly the size asked for, between guards
    descs, ptrs = plan._describe()
    size = ctypes.c_size_t()
    assert tsr.lib().tsr_dense_plan_workspace_bytes(plan.ctx, ctypes.byref(size)) == 0
    end = 256 + size.value
    room = torch.full((end + 4096,), 0xA5, dtype=torch.uint8, device="cuda")
    assert room.data_ptr() % 256 == 0
    assert tsr.lib().tsr_dense_plan_bind(plan.ctx, (tsr.DensePtrs * 1)(*ptrs), 1, room.data_ptr() + 256, size.value) == 0
    for t in (1, 2):
        plan.step(hyper(t), rounding=rounding, seed=t)
        plan.grad_norm(1.0)
    assert abs(float(plan.grad_norm()[0]) / float(one.grad_norm()[0]) - 1) <= 12 * 2.0 ** -24    # another order of summation
    assert torch.equal(p, ref) and torch.equal(g, g0)
    for a, b in zip(plan.states[0], one.states[0]):
        assert torch.equal(bits(a), bits(b))
    # converted on from there
    other = torch.float32 if kind == F8 else F8
    (want, _), (got, other_guards) = state(n, other, 0, 0), state(n, other, *offsets[::-1])
    tsr.DensePlan(None, None, states=[want]).copy_state(one)
    tsr.DensePlan(None, None, states=[got]).copy_state(plan)
    for a, b in zip(got, want):
        assert torch.equal(bits(a), bits(b))
    assert guards() and other_guards()
    assert bool((room[:256] == 0xA5).all()) and bool((room[end:] == 0xA5).all())


@pytest.mark.parametrize("pitch", [0, 3])
@pytest.mark.parametrize("rounding", [0, 1])
@pytest.mark.parametrize("kind", [torch.float32, F8])
@pytest.mark.parametrize("pd,gd", [(torch.float32, torch.float32), (torch.bfloat16, torch.bfloat16), (torch.bfloat16, torch.float32), (torch.float32, torch.bfloat16)])
def test_moments_at_every_alignment(tsr, pd, gd, kind, rounding, pitch):
    for rows, cols in ((1, 5000), (12, 600), (70, 33), (3, 1)):
        for k in range(1, 8):
            compare(tsr, rows, cols, kind, pd, gd, (k, (3 * k + 1) % 8), pitch, rounding)


@pytest.mark.parametrize("rows,cols,pitch", [(1, 4_000_077, 0), (2001, 2000, 0), (2001, 2000, 8), (130_000, 31, 1)])
@pytest.mark.parametrize("kind", [torch.float32, F8])
@pytest.mark.parametrize("pd", [torch.float32, torch.bfloat16])
def test_moments_off_their_alignment_in_millions_of_elements(tsr, pd, kind, rows, cols, pitch):
    """Enough for several blocks a warp and for thousands of entries in the plan's table."""
    for offsets in ((1, 1), (0, 3)):
        compare(tsr, rows, cols, kind, pd, torch.bfloat16, offsets, pitch, 1)


@pytest.mark.parametrize("kind", [torch.float32, F8])
def test_a_pitch_beyond_32_bits(tsr, kind):
    """Rows 2^30 elements and more apart: chunks of eight blocks, too."""
    if torch.cuda.mem_get_info()[0] < 40 << 30:
        pytest.skip("needs 40 GB of free device memory")
    for rows, cols in ((2, 3_000_000), (5, 300)):
        compare(tsr, rows, cols, kind, torch.bfloat16, torch.bfloat16, (0, 0), (1 << 30) - cols + (rows == 2), 1)

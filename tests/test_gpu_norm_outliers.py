"""Norms of rows with single large entries, and of rows whose entries are all alike, in every form of the forward kernels."""
import pytest
import torch

import layer_model as lm

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def tsr():
    import paper_2602_08007_b200 as t
    return t


def make(rows, cols, dtype, seed, pitch=None, shift=0):
    """Normal entries; rows of `pitch` entries that start `shift` entries into their buffer, surrounded by NaN."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    ld = cols if pitch is None else pitch
    flat = torch.full((rows * ld + shift + 64,), float("nan"), dtype=dtype, device="cuda")
    t = torch.as_strided(flat, (rows, cols), (ld, 1), shift)
    t.copy_(torch.randn(rows, cols, generator=gen, device="cuda"))
    return t


# rows per warp 8, 4, 2, 1; units per lane 1 to 8; teams of 2, 4 and 8 warps; rows read several times
COLS = [2, 3, 24, 100, 128, 500, 1024, 2047, 2048, 2500, 4096, 5461, 8192, 16385]


def layout(name, cols):
    return {"whole": (None, 0), "pitched": (cols + 3, 1)}[name]


@pytest.mark.parametrize("where", ["first", "last", "first unit"])
@pytest.mark.parametrize("lies", ["whole", "pitched", "apart"])
@pytest.mark.parametrize("dt", [F32, BF])
@pytest.mark.parametrize("cols", COLS)
def test_a_large_entry_costs_the_others_nothing(tsr, cols, dt, lies, where):
    """First entries of 1e2 to 1e5 deviations of the others (an outlier channel), within the bounds that rows without them keep.  "apart": y starts at
    another place in 16 bytes than x, which takes the entry-by-entry kernel."""
    pitch, shift = layout("whole" if lies == "apart" else lies, cols)
    x = make(24, cols, dt, 1, pitch, shift)
    at = {"first": slice(0, 1), "last": slice(cols - 1, cols), "first unit": slice(0, min(8, cols))}[where]
    size = torch.tensor([1e2, -3e2, 1.2e3, -1e4, 1.2e4, 1e5], device="cuda").repeat(4)[:, None]
    x[:, at] = (size * (1 + 0.01 * x[:, at].float())).to(dt)
    w, b = make(1, cols, F32, 2)[0], make(1, cols, F32, 3)[0]
    out = make(24, cols, dt, 4, cols + 1, 3) if lies == "apart" else None
    y, stats = tsr.norm_forward(x, w, b, out=out)
    want, sy, mu, smu, rstd, srstd = lm.norm(x, w, b)
    lm.close(stats[:, :1], mu, smu)
    lm.close(stats[:, 1:], rstd, srstd)
    lm.close(y, want, sy)


@pytest.mark.parametrize("cols", [24, 2048, 5461, 8192, 16385])
def test_statistics_to_their_last_digits(tsr, cols):
    """Mean and deviation of FP32 rows with a first entry of 3e4 deviations.  The mean: half a step of itself, and the sum of the distances from the first
    approximation, of at most 64 additions on any path, 2^-18 of their mean size.  (Distances from the first entry were rounded to 2^-24 of 3e4 each.)"""
    x = make(32, cols, F32, 5)
    x[:, 0] = 3e4
    _, stats = tsr.norm_forward(x)
    d = x.double() - x.double().mean(1, keepdim=True)
    lm.close(stats[:, :1], x.double().mean(1, keepdim=True), 2.0 ** -18 * d.abs().mean(1, keepdim=True) * (1 + 2.0 ** -10))


@pytest.mark.parametrize("center", [True, False])
@pytest.mark.parametrize("lies", ["whole", "pitched", "apart"])
@pytest.mark.parametrize("dt", [F32, BF])
@pytest.mark.parametrize("cols", COLS)
def test_rows_of_equal_entries(tsr, cols, dt, lies, center):
    """Their variance is zero, whatever the entry: y is the bias to the bit, the mean the entry, the deviation that of eps."""
    pitch, shift = layout("whole" if lies == "apart" else lies, cols)
    x = make(7, cols, dt, 1, pitch, shift)
    x.copy_(torch.tensor([0.0, 0.1, -3.7, 1e5 / 3, -1e18, 1e-30, 65504.0], device="cuda")[:, None].expand(7, cols))
    b = make(1, cols, F32, 3)[0]
    out = make(7, cols, dt, 4, cols + 1, 3) if lies == "apart" else None
    y, stats = tsr.norm_forward(x, None, b, eps=1e-6, center=center, out=out)
    if center:
        assert torch.equal(y, b.to(dt).expand(7, cols)) and torch.equal(stats[:, 0], x[:, 0].float())
        assert float((stats[:, 1] * 1e-3 - 1).abs().max()) <= 2.0 ** -20
    else:      # (FP32 holds sums up to 3.4e38: 340 squares of 1e18)
        some = [i for i in range(7) if i != 4 or cols < 340]
        lm.close(y[some], *[t[some] for t in lm.norm(x, None, b, 1e-6, False)[:2]])


def test_a_row_with_an_infinity_has_that_mean(tsr):
    for cols in (24, 100, 2048, 5461, 16385):
        x = make(4, cols, F32, 1)
        x[0, 0], x[1, 5], x[2, cols - 1], x[3, 3] = float("inf"), float("-inf"), float("inf"), float("nan")
        y, stats = tsr.norm_forward(x)
        assert torch.isnan(y).all() and torch.isnan(stats[:, 1]).all()
        assert torch.equal(stats[:3, 0], torch.tensor([float("inf"), float("-inf"), float("inf")], device="cuda")) and torch.isnan(stats[3, 0])

"""Norms over rows against their formulas in 64 bits: types, widths of every kernel, odd sizes, pitches, alignment, gradients."""
import pytest
import torch

import layer_model as lm

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def tsr():
    import paper_2602_08007_b200 as t
    return t


def make(rows, cols, dtype, seed, sigma=1.0, mean=0.0, pitch=None, shift=0):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    ld = cols if pitch is None else pitch
    flat = torch.full((rows * ld + shift + 64,), float("nan"), dtype=dtype, device="cuda")
    t = torch.as_strided(flat, (rows, cols), (ld, 1), shift)
    t.copy_(torch.randn(rows, cols, generator=gen, device="cuda") * sigma + mean)
    return t


# widths at the borders of the kernels, odd ones, one entry
SIZES = [(1, 1), (3, 7), (64, 512), (33, 256), (17, 257), (9, 1000), (5, 1024), (40, 2048), (6, 2049), (7, 5461), (4, 8192), (3, 8200), (2, 16384), (3, 16385), (2, 40000), (1000, 24), (3000, 333)]


@pytest.mark.parametrize("center", [True, False])
@pytest.mark.parametrize("layout", ["whole", "pitched", "shifted"])
@pytest.mark.parametrize("dt", [BF, F32])
@pytest.mark.parametrize("rows,cols", SIZES)
def test_forward_and_backward(tsr, rows, cols, dt, layout, center):
    pitch, shift = {"whole": (None, 0), "pitched": ((cols + 15) // 8 * 8, 8), "shifted": (cols + 3, 1)}[layout]
    x = make(rows, cols, dt, 1, 2.0, 0.5, pitch, shift)
    w, b = (make(1, cols, F32 if layout == "whole" else BF, k)[0] for k in (2, 3))
    out = make(rows, cols, dt, 4, pitch=pitch, shift=shift)
    y, stats = tsr.norm_forward(x, w, b, eps=1e-5, center=center, out=out)
    want, sy, mu, smu, rstd, srstd = lm.norm(x, w, b, 1e-5, center)
    lm.close(y, want, sy)
    lm.close(stats[:, :1], mu, smu)
    lm.close(stats[:, 1:], rstd, srstd)
    dy, dx = make(rows, cols, dt, 5, 0.01, pitch=pitch, shift=shift), make(rows, cols, dt, 6, pitch=pitch, shift=shift)
    gw, gb = (make(1, cols, BF if layout == "shifted" else F32, k)[0] for k in (7, 8))
    accumulate = layout != "whole"
    w0, b0 = (t.double() if accumulate else torch.zeros(cols, dtype=torch.float64, device="cuda") for t in (gw, gb))
    rx, rw, rb = tsr.norm_backward(dy, x, w, stats, center=center, dx=dx, dweight=gw, dbias=gb, accumulate=accumulate)
    (ex, sx), (ew, sw), (eb, sb) = lm.norm_grads(dy, x, w, stats, center)
    lm.close(rx, ex, sx)
    lm.close(rw, ew + w0, sw + 2.0 ** -23 * ((ew + w0).abs() + w0.abs()))
    lm.close(rb, eb + b0, sb + 2.0 ** -23 * ((eb + b0).abs() + b0.abs()))
    for t in (out, dx):
        if pitch:
            assert torch.isnan(torch.as_strided(t, (rows, pitch - cols), (pitch, 1), shift + cols)).all()


# every form of the row kernels (lanes per row, units per lane, teams of warps), over many turns of their rings, with groups that run out earlier than others
MANY = [(30011, 8), (30011, 9), (30011, 31), (20011, 64), (20011, 100), (20011, 129), (20011, 257), (12011, 500), (9011, 1000), (9011, 1023), (6011, 2047), (6011, 2048),
        (5011, 2500), (4011, 3500), (3011, 4096), (3011, 4500), (3011, 5461), (2511, 7000), (2011, 8192), (2011, 8190), (1511, 10001), (1511, 12000), (1211, 16001)]


@pytest.mark.parametrize("dt", [BF, F32])
@pytest.mark.parametrize("rows,cols", MANY)
def test_many_rows(tsr, rows, cols, dt):
    x, dy, w, b = make(rows, cols, dt, 1, 2.0, 0.5), make(rows, cols, dt, 2), make(1, cols, F32, 3)[0], make(1, cols, F32, 4)[0]
    for center in (True, False):
        y, stats = tsr.norm_forward(x, w, b, center=center)
        want, sy, mu, smu, rstd, srstd = lm.norm(x, w, b, 1e-5, center)
        lm.close(y, want, sy)
        lm.close(stats[:, :1], mu, smu)
        lm.close(stats[:, 1:], rstd, srstd)
        rx, rw, rb = tsr.norm_backward(dy, x, w, stats, center=center, bias=center)
        (ex, sx), (ew, sw), (eb, sb) = lm.norm_grads(dy, x, w, stats, center)
        lm.close(rx, ex, sx)
        lm.close(rw, ew, sw)
        if center:
            lm.close(rb, eb, sb)
    assert tsr.layer_poll_status() == tsr.TSR_OK


@pytest.mark.parametrize("rows,cols", [(50, 96), (20, 3000), (3, 20000)])
def test_parts_that_are_left_out(tsr, rows, cols):
    x, dy = make(rows, cols, F32, 1), make(rows, cols, F32, 2)
    y, stats = tsr.norm_forward(x)
    lm.close(y, *lm.norm(x)[:2])
    w = make(1, cols, F32, 3)[0]
    (ex, sx), (ew, sw), (eb, sb) = lm.norm_grads(dy, x, w, stats)
    for want_dx in (True, False):
        for want_dw in (True, False):
            for bias in (True, False):
                dx, dw, db = tsr.norm_backward(dy, x, w, stats, bias=bias, want_dx=want_dx, want_dweight=want_dw)
                assert (dx is not None, dw is not None, db is not None) == (want_dx, want_dw, bias)
                if want_dx:
                    lm.close(dx, ex, sx)
                if want_dw:
                    lm.close(dw, ew, sw)
                if bias:
                    lm.close(db, eb, sb)


@pytest.mark.parametrize("cols", [100, 1111, 20000])
def test_in_place(tsr, cols):
    x, dy = make(30, cols, BF, 1), make(30, cols, BF, 2)
    y, stats = tsr.norm_forward(x)
    again = x.clone()
    z, _ = tsr.norm_forward(again, out=again)
    assert z is again and torch.equal(z, y)
    dx, _, _ = tsr.norm_backward(dy, x, None, stats)
    own = dy.clone()
    tsr.norm_backward(own, x, None, stats, dx=own, bias=False)
    assert torch.equal(own, dx)


def test_large_mean_keeps_its_digits(tsr):
    """The squares are of distances from the mean: a mean of 1000 deviations costs no more than the rounding of the entries."""
    x = make(40, 2000, F32, 1, 1.0, 1000.0)
    y, stats = tsr.norm_forward(x)
    want, sy, mu, _, rstd, _ = lm.norm(x)
    assert float((stats[:, 1:].double() / rstd - 1).abs().max()) < 1e-5
    lm.close(y, want, sy)


def test_rows_that_are_zero_huge_or_not_finite(tsr):
    x = make(6, 300, F32, 1)
    x[0] = 0.0
    x[1] = 1e18
    x[2, 5] = float("nan")
    x[3, 7] = float("inf")
    y, stats = tsr.norm_forward(x, eps=1e-6)
    assert (y[0] == 0).all() and (y[1] == 0).all()
    assert torch.isnan(y[2]).all() and torch.isnan(y[3]).all()
    lm.close(y[4:], *[t[4:] for t in lm.norm(x, eps=1e-6)[:2]])


def test_empty(tsr):
    for shape in [(0, 8), (5, 0), (0, 0)]:
        x = torch.empty(shape, device="cuda")
        w = torch.ones(shape[1], device="cuda")
        y, stats = tsr.norm_forward(x, w, w)
        assert y.shape == x.shape and tuple(stats.shape) == (shape[0], 2)
        dx, dw, db = tsr.norm_backward(x, x, w, stats)
        assert dx.shape == x.shape and (dw == 0).all() and (db == 0).all() and dw.shape == w.shape


def test_same_bits_every_time(tsr):
    x, dy, w = make(2500, 1376, BF, 1), make(2500, 1376, BF, 2), make(1, 1376, F32, 3)[0]
    y, stats = tsr.norm_forward(x, w, w)
    first = tsr.norm_backward(dy, x, w, stats)
    for _ in range(3):
        for a, b in zip(first, tsr.norm_backward(dy, x, w, stats)):
            assert torch.equal(a, b)

"""Dropout: exactly the entries that the words say, in every layout, alone and inside a linear layer."""
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
    gen = torch.Generator(device="cuda").manual_seed(seed)
    ld = cols if pitch is None else pitch
    flat = torch.full((rows * ld + shift + 64,), float("nan"), dtype=dtype, device="cuda")
    t = torch.as_strided(flat, (rows, cols), (ld, 1), shift)
    t.copy_(torch.randn(rows, cols, generator=gen, device="cuda"))
    return t


@pytest.mark.parametrize("layout", ["whole", "pitched", "shifted"])
@pytest.mark.parametrize("dt", [BF, F32])
@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 100001), (64, 512), (33, 45), (3000, 8), (700, 1376), (5000, 1)])
def test_entries(tsr, rows, cols, dt, layout):
    pitch, shift = {"whole": (None, 0), "pitched": ((cols + 15) // 8 * 8, 8), "shifted": (cols + 3, 1)}[layout]
    x, res, out = make(rows, cols, dt, 1, pitch, shift), make(rows, cols, dt, 2, pitch, shift), make(rows, cols, dt, 3, pitch, shift)
    for p in (0.0, 0.1, 0.5, 1.0):
        d = tsr.Dropout(p, 2 ** 63 + 12345, 2 ** 40 + 7)
        for r in (None, res):
            y = tsr.dropout_forward(x, d, residual=r, out=out)
            want = lm.drop(x.double(), d)
            lm.close(y, want if r is None else want + res.double(), 2.0 ** -23 * want.abs())
            if pitch:
                assert torch.isnan(torch.as_strided(out, (rows, pitch - cols), (pitch, 1), shift + cols)).all()
    d = tsr.Dropout(0.3, 5)
    assert torch.equal(tsr.dropout_backward(x, d), tsr.dropout_forward(x, d))


def test_far_rows_and_offsets(tsr):
    """The upper words of offset and row count: two rows whose pitch spans 2^32 entries, and an offset that wraps."""
    flat = torch.zeros(2 ** 32 + 4096, dtype=BF, device="cuda")
    x = torch.as_strided(flat, (2, 1000), (2 ** 32, 1), 0)
    x.fill_(1.0)
    d = tsr.Dropout(0.5, 1, 2)
    y = tsr.dropout_forward(x, d)
    lm.close(y, lm.drop(torch.ones(2, 1000, dtype=torch.float64, device="cuda"), d), torch.zeros((), dtype=torch.float64, device="cuda"))
    step = torch.tensor([2], device="cuda")
    a = tsr.dropout_forward(x, tsr.Dropout(0.5, 1, 2 ** 64 - 1, step))
    b = tsr.dropout_forward(x, tsr.Dropout(0.5, 1, 1))
    assert torch.equal(a, b)


def test_what_falls_is_zero(tsr):
    x = torch.full((50, 64), float("nan"), device="cuda")
    x[::2] = float("inf")
    d = tsr.Dropout(0.25, 9)
    y = tsr.dropout_forward(x, d)
    keep = torch.from_numpy(lm.kept(50, 64, 0.25, 9, 0)).cuda()
    assert (y[~keep] == 0).all() and not torch.isfinite(y[keep]).any()


def test_rates_and_independence(tsr):
    """Shares of entries that fall, alone and together with a neighbour, the next row, another offset, within five deviations."""
    n = 1 << 22
    x = torch.ones(2048, 2048, device="cuda")
    for p in (0.1, 0.5):
        a = tsr.dropout_forward(x, tsr.Dropout(p, 7, 0)) == 0
        b = tsr.dropout_forward(x, tsr.Dropout(p, 7, 1)) == 0
        c = tsr.dropout_forward(x, tsr.Dropout(p, 8, 0)) == 0
        for u, v in ((a[:, 1:], a[:, :-1]), (a[1:], a[:-1]), (a[:, 2:], a[:, :-2]), (a, b), (a, c)):
            share = float((u & v).double().mean())
            assert abs(share - p * p) < 5 * (p * p * (1 - p * p) / u.numel()) ** 0.5 + 2 ** -15
        assert abs(float(a.double().mean()) - p) < 5 * (p * (1 - p) / n) ** 0.5 + 2 ** -16


def test_linear_layers_draw_the_same_entries(tsr):
    """A layer's dropout is the operator's own: every tile shape, split sums, and the backward pass."""
    for T, I, O in [(300, 64, 400), (1, 2048, 256), (2, 8192, 64), (77, 40, 91)]:
        x = make(T, I, BF, 1)
        w = torch.zeros(O, I, dtype=BF, device="cuda")
        b = torch.ones(O, device="cuda")
        d = tsr.Dropout(0.4, 31, 17)
        y, _ = tsr.linear_forward(x, w, b, dropout=d)
        assert torch.equal(y, tsr.dropout_forward(torch.ones(T, O, dtype=BF, device="cuda"), d))
        db = torch.empty(O, device="cuda")
        tsr.linear_backward(torch.ones(T, O, dtype=BF, device="cuda"), x, w, dropout=d, dbias=db, want_dx=False, want_dweight=False)
        want = lm.drop(torch.ones(T, O, dtype=torch.float64, device="cuda"), d).sum(0)
        lm.close(db, want, 2.0 ** -15 * want.abs())

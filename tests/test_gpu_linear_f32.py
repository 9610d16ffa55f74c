"""What an FP32 layer keeps of its 24 bits: each product of parts on its own, the size of the error as a whole, infinities."""
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


# An operand x is held as BF16 parts p1 + p2 + p3.  Two neighbours in K whose products cancel but for one product of parts:
#   (first x, first w), (second x, second w), what is left of the sum
PARTS = {
    "p1 q2": ((1.0, 1 + 2.0 ** -10), (-1.0, 1.0), 2.0 ** -10),
    "p2 q1": ((1 + 2.0 ** -10, 1.0), (1.0, -1.0), 2.0 ** -10),
    "p2 q2": ((1 + 2.0 ** -10, 1 + 2.0 ** -10), (-1.0, 1 + 2.0 ** -9), 2.0 ** -20),
    "p1 q3": ((1.0, 1 + 2.0 ** -10 + 2.0 ** -20), (-1.0, 1 + 2.0 ** -10), 2.0 ** -20),
    "p3 q1": ((1 + 2.0 ** -10 + 2.0 ** -20, 1.0), (1 + 2.0 ** -10, -1.0), 2.0 ** -20),
}


def planted(parts, M, N, K, k, device="cuda"):
    """A (M x K) and B (N x K), zero but for columns k and k + 1 (k even), each row scaled by a power of two of its own; and A B^T, exact in FP32."""
    (x0, w0), (x1, w1), left = PARTS[parts]
    s = torch.pow(2.0, torch.arange(M, device=device).float() % 7 - 3)
    t = torch.pow(2.0, torch.arange(N, device=device).float() % 5 - 2)
    A, B = torch.zeros(M, K, device=device), torch.zeros(N, K, device=device)
    A[:, k], A[:, k + 1], B[:, k], B[:, k + 1] = x0 * s, x1 * s, w0 * t, w1 * t
    return A, B, left * s[:, None] * t[None, :]


# one CTA and pairs, tiles of every width, whole and split K, K blocks and chunks of 128 that are not whole
SHAPES = [(100, 40, 40), (130, 70, 600), (300, 200, 1000), (1000, 264, 130), (2500, 1376, 512), (128, 64, 5462)]


@pytest.mark.parametrize("M,N,K", SHAPES)
@pytest.mark.parametrize("parts", sorted(PARTS))
def test_each_product_of_parts(tsr, parts, M, N, K):
    """The result is exact: the terms are powers of two, at most 2^21 apart, which an FP32 accumulator holds."""
    for k in sorted({0, 30, K // 2 // 2 * 2, (K - 2) // 2 * 2}):
        A, B, want = planted(parts, M, N, K, k)
        y, _ = tsr.linear_forward(A, B)                                   # both K-major
        assert torch.equal(y, want), ("forward", k)
        none = torch.zeros(1, device="cuda")
        dx, _, _ = tsr.linear_backward(A, None, B.t().contiguous(), want_dweight=False)     # dz K-major, the weight MN-major
        assert torch.equal(dx, want), ("dx", k)
        _, dw, _ = tsr.linear_backward(A.t().contiguous(), B.t().contiguous(), none.expand(M, N).contiguous(), want_dx=False)     # both MN-major
        assert torch.equal(dw, want), ("dweight", k)


@pytest.mark.parametrize("M,N,K", SHAPES + [(600, 500, 4096)])
def test_size_of_the_error(tsr, M, N, K):
    """Operands and products of parts lose at most 2^-25.  Within 128 entries of K there are 48 additions to the tensor cores' accumulator; each cuts off up to
    2^-23 of it, half of that on average, while it has two thirds of its last size on average: 48 x 2^-24 x 2/3 = 32 x 2^-24 of the root of the sum of
    squares.  (Without the third parts it would be 74 x 2^-24.)  The accumulators themselves are added to nearest."""
    A, B = normal(M, K, seed=1), normal(N, K, seed=2, sigma=0.1)

    def check(got, a, b):
        off = (got.double() - a.double() @ b.double().t()).square().sum().sqrt()
        size = ((a.double() ** 2) @ (b.double() ** 2).t()).sum().sqrt()
        assert float(off / size) <= 32 * 2.0 ** -24, float(off / size * 2.0 ** 24)

    check(tsr.linear_forward(A, B)[0], A, B)
    check(tsr.linear_backward(A, None, B.t().contiguous(), want_dweight=False)[0], A, B)
    check(tsr.linear_backward(A.t().contiguous(), B.t().contiguous(), torch.empty(M, N, device="cuda"), want_dx=False)[1], A, B)


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

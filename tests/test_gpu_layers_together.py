"""The layer operators as they are used: in a row, under autograd, into the optimizer's gradients, on other streams, in captured graphs."""
import copy
import importlib.util
import io
import os

import pytest
import torch

import layer_model as lm

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def tsr():
    import paper_2602_08007_b200 as t
    return t


def normal(*shape, dtype=F32, seed=1, sigma=1.0):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn(*shape, generator=gen, device="cuda") * sigma).to(dtype)


def block64(x, nw, nb, w1, b1, w2, b2, d1, d2):
    """norm -> linear with GELU and dropout -> linear with dropout and residual, in 64 bits, for torch to differentiate."""
    h = (x - x.mean(1, keepdim=True)) / torch.sqrt(x.var(1, unbiased=False, keepdim=True) + 1e-5) * nw + nb
    a = lm.drop(torch.nn.functional.gelu(h @ w1.t() + b1), d1)
    return x + lm.drop(a @ w2.t() + b2, d2)


def test_a_feed_forward_block_in_fp32(tsr):
    """Forward, and every gradient against the formula's and against differences.  FP32 keeps 2^-20 of the largest intermediate here: tolerance
    2^-16 of the largest value of each result."""
    T, H, F = 200, 96, 264
    args = [normal(T, H, seed=1), 1 + normal(H, seed=2, sigma=0.1), normal(H, seed=3, sigma=0.1), normal(F, H, seed=4, sigma=0.1), normal(F, seed=5, sigma=0.1),
            normal(H, F, seed=6, sigma=0.1), normal(H, seed=7, sigma=0.1)]
    d1, d2 = tsr.Dropout(0.2, 11, 3), tsr.Dropout(0.1, 11, 4)
    leaves = [a.clone().requires_grad_() for a in args]
    x, nw, nb, w1, b1, w2, b2 = leaves
    y = tsr.linear(tsr.linear(tsr.layer_norm(x, nw, nb), w1, b1, activation="gelu", dropout=d1), w2, b2, dropout=d2, residual=x)
    up = normal(T, H, seed=8)
    y.backward(up)
    exact = [a.double().requires_grad_() for a in args]
    z = block64(*exact, d1, d2)
    z.backward(up.double())
    assert float((y.double() - z).detach().abs().max()) <= 2.0 ** -16 * float(z.detach().abs().max())
    for name, a, b in zip(["x", "norm weight", "norm bias", "w1", "b1", "w2", "b2"], leaves, exact):
        assert float((a.grad.double() - b.grad).abs().max()) <= 2.0 ** -16 * float(b.grad.abs().max()), name
    # differences of the formula along a direction: central, step 1e-6 in 64 bits, off by its square and by 1e-16 / 1e-6 of the values
    with torch.no_grad():
        for i, a in enumerate(leaves):
            v = normal(*a.shape, seed=20 + i).double()
            plus, minus = ([e.detach() + (s * 1e-6 * v if j == i else 0) for j, e in enumerate(exact)] for s in (1, -1))
            slope = ((block64(*plus, d1, d2) - block64(*minus, d1, d2)) * up.double()).sum() / 2e-6
            size = (a.grad.double().abs() * v.abs()).sum()
            assert abs(float((a.grad.double() * v).sum() - slope)) <= 2.0 ** -14 * float(size) + 1e-6


def test_the_same_block_in_bf16_step_by_step(tsr):
    """Each operator against its own formula on what the one before left."""
    T, H, F = 300, 128, 520
    x, nw = normal(T, H, dtype=BF, seed=1), 1 + normal(H, seed=2, sigma=0.1)
    w1, w2, b1 = normal(F, H, dtype=BF, seed=3, sigma=0.1), normal(H, F, dtype=BF, seed=4, sigma=0.1), normal(F, dtype=BF, seed=5)
    d = tsr.Dropout(0.1, 5, 6)
    h, stats = tsr.norm_forward(x, nw, None, center=False)
    lm.close(h, *lm.norm(x, nw, None, 1e-5, False)[:2])
    a, pre = tsr.linear_forward(h, w1, b1, activation="silu", keep_pre=True)
    want, wz, sa, sz = lm.linear(h, w1, b1, "silu")
    lm.close(a, want, sa), lm.close(pre, wz, sz)
    y, _ = tsr.linear_forward(a, w2, dropout=d, residual=x)
    want, _, sy, _ = lm.linear(a, w2, None, "none", d, x)
    lm.close(y, want, sy)
    dy = normal(T, H, dtype=BF, seed=7)
    da, dw2, _ = tsr.linear_backward(dy, a, w2, dropout=d)
    for got, (e, s) in zip((da, dw2), lm.linear_grads(dy, a, w2, None, "none", d)):
        lm.close(got, e, s)
    gb = torch.empty(F, device="cuda")
    dh, dw1, db1 = tsr.linear_backward(da, h, w1, pre=pre, activation="silu", dbias=gb)
    for got, (e, s) in zip((dh, dw1, db1), lm.linear_grads(da, h, w1, pre, "silu")):
        lm.close(got, e, s)
    dx, dn, _ = tsr.norm_backward(dh, x, nw, stats, center=False, bias=False)
    for got, (e, s) in zip((dx, dn), lm.norm_grads(dh, x, nw, stats, False)):
        lm.close(got, e, s)


def test_gradients_that_autograd_brings(tsr):
    """Expanded upstream gradients, inputs that have to be copied, a bias in BF16, a residual's gradient, inputs that need none."""
    x = normal(48, 64, seed=1).t().requires_grad_()          # (64, 48), columns contiguous
    w = normal(48, 32, seed=2, sigma=0.2).t().contiguous().requires_grad_()
    b = normal(32, dtype=BF, seed=3).requires_grad_()
    res = normal(64, 32, seed=4).requires_grad_()
    tsr.linear(x, w, b, activation="relu", residual=res).sum().backward()
    ex, ew, eb = (t.detach().double().requires_grad_() for t in (x, w, b))
    torch.relu(ex @ ew.t() + eb).sum().backward()
    for got, want in ((x.grad, ex.grad), (w.grad, ew.grad), (b.grad, eb.grad)):
        assert got.dtype in (F32, BF) and float((got.double() - want).abs().max()) <= (2.0 ** -8 if got.dtype == BF else 2.0 ** -18) * float(want.abs().max())
    assert (res.grad == 1).all()
    # only some inputs
    w2 = normal(16, 64, seed=5).requires_grad_()
    tsr.linear(normal(10, 64, seed=6), w2).sum().backward()
    assert w2.grad is not None
    y = tsr.layer_norm(normal(10, 64, seed=7).requires_grad_())
    y.backward(torch.ones(1, device="cuda").expand(10, 64))
    z = normal(9, 24, seed=8).requires_grad_()
    d = tsr.Dropout(0.5, 1)
    tsr.dropout(z, d, residual=z).sum().backward()
    want = 1 + lm.drop(torch.ones(9, 24, dtype=torch.float64, device="cuda"), d)
    assert torch.equal(z.grad.double(), want)
    with torch.no_grad():
        assert not tsr.linear(z, normal(4, 24)).requires_grad


def test_weight_gradients_go_where_the_optimizer_reads_them(tsr):
    """Into the G of TSR blocks (5461 columns at a pitch of 5464), written by the first micro batch and added to by the second; then a step runs on it."""
    shapes = [(256, 320), (192, 5461)]
    plan = tsr.Plan([dict(m=m, n=n, r=32, p=8, q=1, K=0) for m, n in shapes], g_dtype=BF)
    for W, (m, n) in zip(plan.W, shapes):
        W.normal_(0, 0.05)
    # The first write rounds the first sum s1 by up to 2^-8 |s1|.  The second adds s2 to that and rounds again (counted by `close`), so the first
    # error stays as it is, however small s1 + s2 has become: relative to s1, not to the total.
    total, rounded = [0.0, 0.0], [0.0, 0.0]
    for micro in range(2):
        for i, (m, n) in enumerate(shapes):
            w = plan.W[i].to(BF).requires_grad_()
            x, up = normal(130, n, dtype=BF, seed=10 * micro + i), normal(130, m, dtype=BF, seed=20 + 10 * micro + i)
            tsr.linear(x, w, weight_grad=plan.G[i], accumulate=micro > 0).backward(up)
            assert w.grad is None
            total[i] = total[i] + up.double().t() @ x.double()
            mag = up.double().abs().t() @ x.double().abs()
            # 2^-19 of the magnitudes: FP32 accumulation of 130 products
            lm.close(plan.G[i], total[i], rounded[i] + mag * 2.0 ** -19)
            rounded[i] = rounded[i] + 2.0 ** -8 * total[i].abs()
    before = [W.clone() for W in plan.W]
    plan.init_subspace(seed=1)
    plan.step(tsr.make_hyper(1))
    assert plan.poll_status() == [0, 0] and all(not torch.equal(a, b) for a, b in zip(before, plan.W))
    # a weight that is used twice needs accumulate over zeros
    G, w, x = torch.zeros(24, 40, device="cuda"), normal(24, 40, seed=1).requires_grad_(), normal(7, 40, seed=2)
    (tsr.linear(x, w, weight_grad=G, accumulate=True) + 2 * tsr.linear(x, w, weight_grad=G, accumulate=True)).sum().backward()
    assert float((G - 3 * x.sum(0)[None, :]).abs().max()) < 1e-4


def test_streams(tsr):
    """Two calls at once, on torch's current stream and on a given one."""
    xs = [normal(2000, 512, dtype=BF, seed=i) for i in range(2)]
    w, nw, dy = normal(768, 512, dtype=BF, seed=5, sigma=0.1), normal(512, seed=6), normal(2000, 768, dtype=BF, seed=7)
    d = tsr.Dropout(0.1, 3)

    def one(x, stream=None):
        h, stats = tsr.norm_forward(x, nw, nw, stream=stream)
        y, pre = tsr.linear_forward(h, w, activation="gelu", dropout=d, keep_pre=True, stream=stream)
        gb = torch.empty(768, device="cuda")
        g = tsr.linear_backward(dy, h, w, pre=pre, activation="gelu", dropout=d, dbias=gb, stream=stream)
        n = tsr.norm_backward(g[0], x, nw, stats, stream=stream)
        return [h, y, *g, *n, tsr.dropout_forward(x, d, stream=stream)]

    want = [one(x) for x in xs]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = [None, None]
    for rep in range(5):
        for i, s in enumerate(streams):
            if i:
                got[i] = one(xs[i], stream=s)
            else:
                with torch.cuda.stream(s):
                    got[i] = one(xs[i])
    torch.cuda.synchronize()
    for a, b in zip(want, got):
        for u, v in zip(a, b):
            assert torch.equal(u, v)
    assert tsr.layer_poll_status() == tsr.TSR_OK


def test_captured_graphs(tsr):
    """Two graphs of the same calls, replayed side by side; a device word moves the dropout from replay to replay."""
    w, nw = normal(640, 512, dtype=BF, seed=1, sigma=0.1), normal(512, seed=2)
    inputs = [normal(700, 512, dtype=BF, seed=3 + i) for i in range(2)]
    ups = [normal(700, 640, dtype=BF, seed=5 + i) for i in range(2)]
    step = torch.zeros(1, dtype=torch.int64, device="cuda")
    d = tsr.Dropout(0.3, 9, 100, step=step)

    def one(x, dy):
        h, stats = tsr.norm_forward(x, nw)
        y, pre = tsr.linear_forward(h, w, activation="silu", dropout=d, keep_pre=True)
        dh, dw, _ = tsr.linear_backward(dy, h, w, pre=pre, activation="silu", dropout=d)
        return [y, dw, *tsr.norm_backward(dh, x, nw, stats)]

    graphs, held = [], []
    for x, dy in zip(inputs, ups):
        one(x, dy)
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            held.append(one(x, dy))
        graphs.append(g)
    streams = [torch.cuda.Stream() for _ in range(2)]
    for value in (0, 1, 7):
        step.fill_(value)
        for x in inputs:
            x.mul_(1.5)
        want = [one(x, dy) for x, dy in zip(inputs, ups)]
        torch.cuda.synchronize()
        for g, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                g.replay()
        torch.cuda.synchronize()
        for a, b in zip(want, held):
            for u, v in zip(a, b):
                assert torch.equal(u, v)
    assert not torch.equal(tsr.dropout_forward(inputs[0], d), tsr.dropout_forward(inputs[0], tsr.Dropout(0.3, 9, 100)))
    for g in graphs:
        g.reset()


def test_a_capture_beside_a_living_eager_graph_is_refused(tsr):
    x, w = normal(64, 32, seed=1), normal(48, 32, seed=2).requires_grad_()
    eager = tsr.linear(x, w).sum()
    g = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with pytest.raises(RuntimeError, match="still alive"):
        with torch.cuda.graph(g):
            tsr.linear(x, w).sum().backward()
    g.reset()
    eager.backward()
    first = w.grad.clone()
    del eager
    w.grad = None
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        tsr.linear(x, w).sum().backward()
    torch.cuda.current_stream().wait_stream(side)
    w.grad = None
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        tsr.linear(x, w).sum().backward()
    x.mul_(2)
    g.replay()
    torch.cuda.synchronize()
    assert float((w.grad - 2 * first).abs().max()) <= 2.0 ** -16 * float(first.abs().max())
    g.reset()


def test_inference_is_captured_beside_a_living_graph(tsr):
    """What records no graph is not refused; and a leaf that was used stays an ordinary tensor, to copy and to save."""
    x, w = normal(64, 32, seed=1), torch.nn.Parameter(normal(48, 32, seed=2))
    eager = tsr.linear(x, w, activation="gelu")
    g = torch.cuda.CUDAGraph()
    with torch.no_grad():
        tsr.linear(x, w, activation="gelu")
        torch.cuda.synchronize()
        with torch.cuda.graph(g):
            y = tsr.linear(x, w, activation="gelu")
    g.replay()
    assert torch.equal(y, eager.detach())
    g.reset()
    assert torch.equal(copy.deepcopy(w), w)
    buffer = io.BytesIO()
    torch.save(w, buffer)
    buffer.seek(0)
    assert torch.equal(torch.load(buffer, weights_only=True), w)
    eager.sum().backward()


def test_vectors_and_batches(tsr):
    """One dimension, three, none of one of them."""
    w, nw = normal(24, 40, seed=1), normal(40, seed=2)
    x = normal(6, 5, 40, seed=3)
    y = tsr.linear(tsr.rms_norm(x, nw), w)
    assert y.shape == (6, 5, 24)
    for i, j in ((0, 0), (5, 4)):
        one = tsr.linear(tsr.rms_norm(x[i, j], nw), w)
        assert one.shape == (24,) and float((one - y[i, j]).abs().max()) <= 2.0 ** -18 * float(y.abs().max())
    assert tsr.linear(x[:0], w).shape == (0, 5, 24) and tsr.dropout(x[0, 0], tsr.Dropout(0.5, 1)).shape == (40,)
    e = x[:, :0].detach().requires_grad_()
    tsr.layer_norm(e).sum().backward()
    assert e.grad.shape == (6, 0, 40)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    z, _ = tsr.linear_forward(x=x, weight=w, stream=s)
    s.synchronize()
    assert torch.equal(z, tsr.linear_forward(x, w)[0])


@pytest.mark.parametrize("cols,shift", [(9001, 0), (9001, 1), (520, 1), (8193, 0)])
def test_norm_gradient_in_place(tsr, cols, shift):
    """dx replaces dy, on the paths that read dy more than once too (wide rows, matrices that start at different places)."""
    x, dy, w = normal(70, cols, dtype=BF, seed=1), normal(70, cols + 8, dtype=BF, seed=2)[:, shift:shift + cols], normal(cols, seed=3)
    _, stats = tsr.norm_forward(x, w)
    want = [t.clone() for t in tsr.norm_backward(dy, x, w, stats)]
    got = tsr.norm_backward(dy, x, w, stats, dx=dy)
    assert got[0] is dy
    for a, b in zip(want, got):
        assert torch.equal(a, b)


def test_same_bits_every_time(tsr):
    x, w, dy = normal(5000, 256, dtype=BF, seed=1), normal(320, 256, dtype=BF, seed=2), normal(5000, 320, dtype=BF, seed=3)
    gb = torch.empty(320, device="cuda")
    first = [t.clone() for t in tsr.linear_backward(dy, x, w, dbias=gb)]
    for _ in range(4):
        for a, b in zip(first, tsr.linear_backward(dy, x, w, dbias=gb)):
            assert torch.equal(a, b)


def test_many_rows_and_far_offsets(tsr):
    """More rows than a grid dimension takes, and rows that lie more than 2^32 entries apart."""
    x, w = normal(200000, 8, dtype=BF, seed=1), normal(16, 8, dtype=BF, seed=2)
    y, _ = tsr.linear_forward(x, w)
    lm.close(y, *[lm.linear(x, w)[i] for i in (0, 2)])
    h, stats = tsr.norm_forward(x)
    lm.close(h, *lm.norm(x)[:2])
    dx, dw, db = tsr.norm_backward(x, x, None, stats)
    lm.close(dx, *lm.norm_grads(x, x, None, stats)[0])
    flat = torch.zeros(2 ** 32 + 2 ** 13, dtype=BF, device="cuda")
    far = torch.as_strided(flat, (2, 512), (2 ** 32, 1), 0)
    far.copy_(normal(2, 512, seed=3))
    for rows in (far, torch.as_strided(flat, (2, 509), (2 ** 32, 1), 3)):
        h, stats = tsr.norm_forward(rows)
        lm.close(h, *lm.norm(rows)[:2])
        dx, _, db = tsr.norm_backward(rows, rows, None, stats)
        lm.close(dx, *lm.norm_grads(rows, rows, None, stats)[0])
        w = normal(24, rows.shape[1], dtype=BF, seed=4)
        y, _ = tsr.linear_forward(rows, w)
        lm.close(y, *[lm.linear(rows, w)[i] for i in (0, 2)])
        gx, gw, _ = tsr.linear_backward(y, rows, w)
        for got, (e, s) in zip((gx, gw), lm.linear_grads(y, rows, w)):
            lm.close(got, e, s)
    del flat


def test_scratch_of_calls_of_one_size(tsr):
    """The same sizes at another alignment need more scratch (operands are copied), or less again."""
    T, I, O = 130, 264, 200
    flat = normal(T * (I + 8) + O * (I + 8) + 64, dtype=BF, seed=1)
    even = lambda rows, at: torch.as_strided(flat, (rows, I), (I, 1), at)  # noqa: E731
    odd = lambda rows, at: torch.as_strided(flat, (rows, I), (I + 1, 1), at)  # noqa: E731
    dy, gb = normal(T, O, dtype=BF, seed=2), torch.empty(O, device="cuda")
    for view in (even, odd, even, odd):
        x, w = view(T, 0), view(O, T * (I + 8))
        y, _ = tsr.linear_forward(x, w)
        lm.close(y, *[lm.linear(x, w)[i] for i in (0, 2)])
        for got, (e, s) in zip(tsr.linear_backward(dy, x, w, dbias=gb), lm.linear_grads(dy, x, w)):
            lm.close(got, e, s)
    for mx in (even(T, 0), odd(T, 1), even(T, 8)):
        _, stats = tsr.norm_forward(mx)
        up = normal(T, I, dtype=BF, seed=3)
        for got, (e, s) in zip(tsr.norm_backward(up, mx, None, stats, want_dweight=True), lm.norm_grads(up, mx, None, stats)):
            lm.close(got, e, s)


def test_refusals(tsr):
    x, w, v = normal(6, 16), normal(8, 16), normal(16, seed=2)
    y, stats = tsr.norm_forward(x, v)
    bad = [
        lambda: tsr.norm_forward(x.half()), lambda: tsr.norm_forward(x.t()), lambda: tsr.norm_forward(x, v[:8]), lambda: tsr.norm_forward(x, v.double()),
        lambda: tsr.norm_forward(x, v, v.to(BF)), lambda: tsr.norm_forward(x, out=torch.empty(1, 16, device="cuda").expand(6, 16)),
        lambda: tsr.norm_forward(x, out=torch.empty(6, 16)), lambda: tsr.norm_forward(x, v.cpu()),
        lambda: tsr.norm_backward(x.to(BF), x, v, stats), lambda: tsr.norm_backward(x[:5], x, v, stats), lambda: tsr.norm_backward(x, x, v, stats[:5]),
        lambda: tsr.norm_backward(x, x, v, stats.t()), lambda: tsr.norm_backward(x, x, v, stats, accumulate=True),
        lambda: tsr.linear_forward(x, w.t()), lambda: tsr.linear_forward(x, w.to(BF)), lambda: tsr.linear_forward(x, w, v), lambda: tsr.linear_forward(x, w, activation="tanh"),
        lambda: tsr.linear_forward(x, w, residual=x), lambda: tsr.linear_forward(x, w, out=torch.empty(6, 9, device="cuda")), lambda: tsr.linear_forward(x, w[0]),
        lambda: tsr.linear_backward(normal(6, 8), x, w, activation="relu"), lambda: tsr.linear_backward(normal(6, 8), None, w),
        lambda: tsr.linear_backward(normal(6, 8), x, w, accumulate=True), lambda: tsr.linear_backward(normal(6, 8), x, w, dweight=torch.empty(8, 16, device="cuda", dtype=torch.float64)),
        lambda: tsr.linear_backward(normal(6, 8), x, w, dbias=torch.empty(7, device="cuda")), lambda: tsr.linear(x, w, weight_grad=torch.empty(8, 16, device="cuda")),
        lambda: tsr.dropout_forward(x, tsr.Dropout(0.1, 0), residual=x[:3]), lambda: tsr.dropout_forward(x, tsr.Dropout(0.1, 0, step=torch.zeros(2, dtype=torch.int64, device="cuda"))),
    ]
    for k, call in enumerate(bad):
        with pytest.raises(ValueError):
            call()
            pytest.fail("call %d was taken" % k)
    with pytest.raises(tsr.TsrError) as e:
        tsr.norm_forward(x, eps=-1.0)
    assert e.value.status == 1
    with pytest.raises(tsr.TsrError) as e:
        tsr.linear_forward(x, w, activation=9)
    assert e.value.status == 6


def test_the_example_on_the_layer_operators(tsr):
    """Runs with dropout, and its first gradients are those of the plain model without: BF16 activations through four blocks differ by a few
    roundings of each, 2^-8 apiece, so half a per cent of a matrix's gradient norm times sixteen roundings bounds them."""
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "pretrain_small.py")
    spec = importlib.util.spec_from_file_location("pretrain_small", path)
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    kept = {}

    def seen(name):
        def at(t, G, others):
            if t == 1:
                kept[name] = [g.double().clone() for g in list(G) + list(others)]
        return at

    example.train(steps=2, seen=seen("plain"))
    example.train(steps=2, layers=True, seen=seen("layers"))
    for a, b in zip(kept["plain"], kept["layers"]):
        assert float((a - b).norm()) <= 16 * 2.0 ** -8 * float(a.norm())
    losses, norms = example.train(steps=6, layers=True, dropout=0.1)
    assert all(torch.isfinite(torch.tensor(losses + norms)))

"""Linear layers against their formulas in 64 bits: types, activations, epilogue, odd sizes, pitches, alignment, every tile shape and splits of K."""
import pytest
import torch

import layer_model as lm

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def tsr():
    import paper_2602_08007_b200 as t
    return t


def make(shape, dtype, seed, sigma=1.0, pitch=None, shift=0):
    """Normal entries; rows of `pitch` entries that start `shift` entries into their buffer, surrounded by NaN."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    r, c = shape
    ld = c if pitch is None else pitch
    flat = torch.full((r * ld + shift + 64,), float("nan"), dtype=dtype, device="cuda")
    t = torch.as_strided(flat, (r, c), (ld, 1), shift)
    t.copy_(torch.randn(r, c, generator=gen, device="cuda") * sigma)
    return t


def check_forward(tsr, T, I, O, dt=BF, kind="none", p=0.0, bias=True, residual=False, pitched=False, bias_type=F32):
    ldi, ldo, shift = (I + 8 - I % 8, O + 8 - O % 8, 8) if pitched else (None, None, 0)
    x, w = make((T, I), dt, 1, pitch=ldi, shift=shift), make((O, I), dt, 2, 0.1, pitch=ldi, shift=shift)
    b = make((1, O), bias_type, 3)[0] if bias else None
    res = make((T, O), dt, 4, pitch=ldo, shift=shift) if residual else None
    out, pre = (make((T, O), dt, k, pitch=ldo, shift=shift) for k in (5, 6))
    d = tsr.Dropout(p, 0x123456789ABCDEF, 5) if p else None
    y, z = tsr.linear_forward(x, w, b, activation=kind, dropout=d, residual=res, out=out, pre=pre if kind != "none" else None)
    want, wz, sy, sz = lm.linear(x, w, b, kind, d, res)
    lm.close(y, want, sy)
    if kind != "none":
        lm.close(z, wz, sz)
    for t in (out, pre):      # what lies between the rows is left alone
        if pitched:
            assert torch.isnan(torch.as_strided(t, (T, ldo - O), (ldo, 1), shift + O)).all()
    assert tsr.layer_poll_status() == tsr.TSR_OK


SIZES = [(1, 64, 64), (1, 2048, 2048), (7, 33, 45), (128, 64, 256), (129, 72, 264), (300, 200, 1000), (513, 768, 2048), (1000, 1376, 512), (257, 5461, 130), (64, 1, 1), (2, 4096, 8)]


@pytest.mark.parametrize("pitched", [False, True])
@pytest.mark.parametrize("T,I,O", SIZES)
def test_forward_sizes(tsr, T, I, O, pitched):
    check_forward(tsr, T, I, O, pitched=pitched)


@pytest.mark.parametrize("T,I,O", SIZES)
def test_forward_sizes_f32(tsr, T, I, O):
    check_forward(tsr, T, I, O, dt=F32, pitched=O % 2 == 0)


@pytest.mark.parametrize("dt", [BF, F32])
@pytest.mark.parametrize("kind", lm.ACTS)
@pytest.mark.parametrize("T,I,O,pitched", [(200, 160, 328, False), (200, 160, 328, True), (65, 77, 91, False), (2, 8192, 64, False)])
def test_forward_epilogue(tsr, dt, kind, T, I, O, pitched):
    check_forward(tsr, T, I, O, dt=dt, kind=kind, p=0.3, residual=True, pitched=pitched, bias_type=BF)


@pytest.mark.parametrize("dt", [BF, F32])
@pytest.mark.parametrize("pitched", [False, True])
@pytest.mark.parametrize("T", [1, 2, 3, 4, 5, 8])
@pytest.mark.parametrize("I,O", [(1, 1), (7, 33), (250, 100), (2048, 2050), (2047, 512), (5461, 77), (6144, 31), (30001, 9), (64, 20011)])
def test_forward_few_rows(tsr, T, I, O, pitched, dt):
    check_forward(tsr, T, I, O, dt=dt, kind="silu", p=0.2, residual=True, pitched=pitched)


@pytest.mark.parametrize("residual", [False, True])
@pytest.mark.parametrize("bias", [False, True])
@pytest.mark.parametrize("p", [0.0, 0.1, 1.0])
def test_forward_options(tsr, residual, bias, p):
    check_forward(tsr, 140, 96, 200, p=p, bias=bias, residual=residual)


@pytest.mark.parametrize("T,I,O", [(4096, 512, 512), (2048, 2048, 1024), (4096, 256, 5461), (20000, 128, 192), (8192, 64, 2048)])
def test_forward_many_tiles(tsr, T, I, O):
    check_forward(tsr, T, I, O, kind="silu", residual=True)


def check_backward(tsr, T, I, O, dt=BF, kind="none", p=0.0, pitched=False, gw=None, accumulate=False, bias=True, wants=(True, True)):
    ldi, ldo, shift = (I + 8 - I % 8, O + 8 - O % 8, 8) if pitched else (None, None, 0)
    x, w = make((T, I), dt, 1, pitch=ldi, shift=shift), make((O, I), dt, 2, 0.1, pitch=ldi, shift=shift)
    dy, pre = make((T, O), dt, 3, pitch=ldo, shift=shift), make((T, O), dt, 4, 2.0, pitch=ldo, shift=shift)
    dx, g = make((T, I), dt, 5, pitch=ldi, shift=shift), make((O, I), gw or dt, 6, pitch=ldi, shift=shift)
    gb = make((1, O), F32, 7)[0] if bias else None
    g0, gb0 = g.clone(), gb.clone() if bias else None
    d = tsr.Dropout(p, 99, 1 << 33) if p else None
    rx, rw, rb = tsr.linear_backward(dy, x if wants[1] else None, w, pre=pre if kind != "none" else None, activation=kind, dropout=d, dx=dx if wants[0] else None,
                                     dweight=g if wants[1] else None, dbias=gb, accumulate=accumulate, want_dx=wants[0], want_dweight=wants[1])
    (ex, sx), (ew, sw), (eb, sb) = lm.linear_grads(dy, x, w, pre, kind, d)
    if accumulate:
        ew, eb = ew + g0.double(), eb + (gb0.double() if bias else 0)
        sw, sb = sw + 2.0 ** -23 * (ew.abs() + g0.double().abs()), sb + 2.0 ** -23 * (eb.abs() + (gb0.double().abs() if bias else 0))
    if wants[0]:
        lm.close(rx, ex, sx)
    else:
        assert rx is None
    if wants[1]:
        lm.close(rw, ew, sw)
    else:
        assert rw is None
    if bias:
        lm.close(rb, eb, sb)
    assert tsr.layer_poll_status() == tsr.TSR_OK


@pytest.mark.parametrize("pitched", [False, True])
@pytest.mark.parametrize("T,I,O", SIZES)
def test_backward_sizes(tsr, T, I, O, pitched):
    check_backward(tsr, T, I, O, pitched=pitched)


@pytest.mark.parametrize("T,I,O", SIZES)
def test_backward_sizes_f32(tsr, T, I, O):
    check_backward(tsr, T, I, O, dt=F32, pitched=O % 2 == 0)


@pytest.mark.parametrize("dt", [BF, F32])
@pytest.mark.parametrize("kind", lm.ACTS)
@pytest.mark.parametrize("T,I,O,pitched", [(200, 160, 328, False), (200, 160, 328, True), (65, 77, 91, False)])
def test_backward_epilogue(tsr, dt, kind, T, I, O, pitched):
    check_backward(tsr, T, I, O, dt=dt, kind=kind, p=0.3, pitched=pitched)


@pytest.mark.parametrize("gw", [BF, F32])
@pytest.mark.parametrize("T,I,O", [(3000, 512, 512), (260, 264, 72), (100, 131, 67), (0, 40, 24), (20000, 64, 128)])
def test_backward_accumulates_into_given_gradients(tsr, gw, T, I, O):
    check_backward(tsr, T, I, O, gw=gw, accumulate=True, pitched=True)


@pytest.mark.parametrize("accumulate", [False, True])
@pytest.mark.parametrize("T,I,O", [(100, 72, 40), (1000, 520, 264), (64, 2048, 2050), (3000, 129, 65), (9, 5461, 300)])
def test_backward_of_fp32_layers_into_bf16_gradients(tsr, T, I, O, accumulate):
    check_backward(tsr, T, I, O, dt=F32, gw=BF, accumulate=accumulate, pitched=accumulate)


@pytest.mark.parametrize("wants", [(True, False), (False, True), (False, False)])
@pytest.mark.parametrize("kind", ["none", "gelu"])
def test_backward_leaves_out_what_is_not_wanted(tsr, wants, kind):
    check_backward(tsr, 150, 64, 96, kind=kind, wants=wants)


@pytest.mark.parametrize("T,I,O", [(4096, 512, 1376), (8192, 2048, 512), (3000, 5461, 256)])
def test_backward_many_tiles(tsr, T, I, O):
    check_backward(tsr, T, I, O, kind="silu", p=0.1, pitched=True)


@pytest.mark.parametrize("dt", [BF, F32])
def test_empty_sizes(tsr, dt):
    for T, I, O in [(0, 16, 24), (5, 0, 24), (5, 16, 0), (0, 0, 0)]:
        x, w = torch.randn(T, I, device="cuda").to(dt), torch.randn(O, I, device="cuda").to(dt)
        b, res = torch.randn(O, device="cuda"), torch.randn(T, O, device="cuda").to(dt)
        y, pre = tsr.linear_forward(x, w, b, activation="relu", residual=res, keep_pre=True)
        want, wz, sy, sz = lm.linear(x, w, b, "relu", None, res)
        lm.close(y, want, sy), lm.close(pre, wz, sz)
        gb = torch.full((O,), 3.0, device="cuda")
        dx, dw, db = tsr.linear_backward(res, x, w, pre=pre, activation="relu", dbias=gb)
        (ex, sx), (ew, sw), (eb, sb) = lm.linear_grads(res, x, w, pre, "relu")
        lm.close(dx, ex, sx), lm.close(dw, ew, sw), lm.close(db, eb, sb)


def test_batched_inputs_and_residual_in_place(tsr):
    x, w = make((6 * 50, 64), BF, 1).view(6, 50, 64), make((80, 64), BF, 2)
    res = make((300, 80), BF, 3).view(6, 50, 80)
    want, _, sy, _ = lm.linear(x.reshape(300, 64), w, None, "none", None, res.reshape(300, 80))
    y, pre = tsr.linear_forward(x, w, residual=res, out=res)
    assert pre is None and y is res
    lm.close(y.reshape(300, 80), want, sy)


@pytest.mark.parametrize("dt", [BF, F32])
def test_what_is_not_finite(tsr, dt):
    """A NaN reaches its row and nothing else; what falls is zero whatever it was; padding and neighbouring rows never leak in."""
    x, w = make((150, 72), dt, 1), make((96, 72), dt, 2)
    x[7, 3] = float("nan")
    y, _ = tsr.linear_forward(x, w)
    assert torch.isnan(y[7]).all() and torch.isfinite(y[:7]).all() and torch.isfinite(y[8:]).all()
    d = tsr.Dropout(0.5, 3)
    y, _ = tsr.linear_forward(x, w, dropout=d)
    keep = torch.from_numpy(lm.kept(150, 96, 0.5, 3, 0)).cuda()
    assert torch.isnan(y[7][keep[7]]).all() and (y[7][~keep[7]] == 0).all()
    dy, pre = make((150, 96), dt, 4), make((150, 96), dt, 5)
    pre[9] = float("nan")
    dy[11] = float("inf")
    _, _, db = tsr.linear_backward(dy, x, w, pre=pre, activation="silu", dropout=d, dbias=torch.empty(96, device="cuda"), want_dx=False, want_dweight=False)
    assert torch.equal(torch.isnan(db) | torch.isinf(db), keep[9] | keep[11])


def test_f32_values_of_every_size(tsr):
    """Columns over many binary orders: errors stay relative to the products themselves."""
    x, w = make((130, 96), F32, 1), make((70, 96), F32, 2)
    scale = torch.pow(2.0, torch.arange(96, device="cuda", dtype=torch.float32) % 41 - 20)
    x, w = x * scale, w / scale
    want, _, sy, _ = lm.linear(x, w)
    y, _ = tsr.linear_forward(x, w)
    lm.close(y, want, sy)
    x = torch.full((130, 8), 3.0e38, device="cuda")
    w = torch.full((70, 8), 0.125 + 2.0 ** -20, device="cuda")
    y, _ = tsr.linear_forward(x * 0.9, w)
    lm.close(y, *[lm.linear(x * 0.9, w)[i] for i in (0, 2)])

"""What the layer calls refuse, and the layouts they take, without a GPU."""
import ctypes

import numpy as np
import pytest
import torch

import layer_model as lm


@pytest.fixture(scope="module")
def tsr():
    import paper_2602_08007_b200 as t
    from paper_2602_08007_b200 import build as b
    b.build()
    return t


AT = 1 << 20      # an aligned address that no call gets as far as using


def norm_desc(tsr, **kw):
    d = dict(rows=4, cols=8, dtype=0, p_dtype=0, g_dtype=0, center=1, accumulate=0, eps=1e-5)
    d.update(kw)
    return tsr.NormDesc(*d.values())


@pytest.mark.parametrize("change,status", [
    (dict(rows=-1), 2), (dict(cols=-1), 2), (dict(rows=(1 << 40) + 1), 2), (dict(cols=0x7fffffff), 2), (dict(dtype=2), 6), (dict(p_dtype=-1), 6),
    (dict(g_dtype=7), 6), (dict(center=2), 1), (dict(eps=-1.0), 1), (dict(eps=float("nan")), 1), (dict(eps=float("inf")), 1),
])
def test_norm_refuses_descriptions(tsr, change, status):
    L, M = tsr.lib(), tsr.Matrix
    d = norm_desc(tsr, **change)
    size = ctypes.c_size_t()
    assert L.tsr_norm_forward(ctypes.byref(d), M(AT, 1 << 31), None, None, M(AT, 1 << 31), None, None) == status
    assert L.tsr_norm_workspace_bytes(ctypes.byref(d), ctypes.byref(size)) == status
    assert L.tsr_norm_backward(ctypes.byref(d), M(AT, 1 << 31), M(AT, 1 << 31), None, AT, M(AT, 1 << 31), None, None, None, 0, None) == status


def test_norm_refuses_matrices(tsr):
    L, M = tsr.lib(), tsr.Matrix
    d = norm_desc(tsr)
    ok, none = M(AT, 8), M(None, 0)

    def fwd(x=ok, w=None, b=None, y=ok, stats=None):
        return L.tsr_norm_forward(ctypes.byref(d), x, w, b, y, stats, None)

    assert fwd(x=none) == 1 and fwd(y=none) == 1 and fwd(x=M(AT, 7)) == 2 and fwd(y=M(AT, 7)) == 2 and fwd(x=M(AT, 1 << 37)) == 2
    assert fwd(x=M(AT + 2, 8)) == 3 and fwd(w=AT + 1) == 3 and fwd(b=AT + 2) == 3 and fwd(stats=AT + 2) == 3
    assert L.tsr_norm_forward(None, ok, None, None, ok, None, None) == 1

    def bwd(dy=ok, x=ok, w=None, stats=AT, dx=ok, dw=None, db=None, ws=AT, size=1 << 30):
        return L.tsr_norm_backward(ctypes.byref(d), dy, x, w, stats, dx, dw, db, ws, size, None)

    assert bwd(dy=none) == 1 and bwd(x=none) == 1 and bwd(stats=None) == 1 and bwd(dx=M(AT, 7)) == 2
    assert bwd(dw=AT + 2) == 3 and bwd(db=AT + 1) == 3 and bwd(dw=AT, ws=None) == 4 and bwd(dw=AT, size=1) == 4 and bwd(db=AT, ws=AT + 64) == 3
    size = ctypes.c_size_t()
    assert L.tsr_norm_workspace_bytes(ctypes.byref(d), ctypes.byref(size)) == 0 and size.value > 0
    assert L.tsr_norm_workspace_bytes(ctypes.byref(d), None) == 1


@pytest.mark.parametrize("rows", [0, 1, 5, 1000, 1 << 30])
@pytest.mark.parametrize("cols", [0, 1, 7, 8, 511, 2048, 4097, 8192, 8193, 100000])
@pytest.mark.parametrize("dtype", [0, 1])
def test_norm_scratch_of_any_size(tsr, rows, cols, dtype):
    size = ctypes.c_size_t()
    assert tsr.lib().tsr_norm_workspace_bytes(ctypes.byref(norm_desc(tsr, rows=rows, cols=cols, dtype=dtype)), ctypes.byref(size)) == 0
    assert (size.value >= 8 * cols and size.value <= 8 * cols * 148 * 24) if cols else size.value == 0


def linear_desc(tsr, drop=(0.0, 0, 0, 0, None), **kw):
    d = dict(rows=100, ins=8, outs=16, dtype=1, b_dtype=0, gw_dtype=0, gb_dtype=0, activation=0, accumulate=0)
    d.update(kw)
    return tsr.LinearDesc(*d.values(), tsr.DropoutDesc(*drop))


@pytest.mark.parametrize("change,status", [
    (dict(rows=-1), 2), (dict(ins=-1), 2), (dict(outs=-1), 2), (dict(rows=0x7fffffff), 2), (dict(rows=1 << 30, dtype=0), 2), (dict(dtype=2), 6), (dict(b_dtype=2), 6),
    (dict(gw_dtype=-1), 6), (dict(gb_dtype=3), 6), (dict(activation=5), 6), (dict(activation=-1), 6), (dict(drop=(-0.1, 0, 0, 0, None)), 1),
    (dict(drop=(1.5, 0, 0, 0, None)), 1), (dict(drop=(float("nan"), 0, 0, 0, None)), 1),
])
def test_linear_refuses_descriptions(tsr, change, status):
    L, M = tsr.lib(), tsr.Matrix
    d, size = linear_desc(tsr, **change), ctypes.c_size_t()
    m = M(AT, 1 << 32)
    io, gr = tsr.LinearIO(m, m, M(None, 0), M(None, 0), m, None), tsr.LinearGrads(m, m, m, m, m, m, None)
    for call, args in ((L.tsr_linear_forward_bytes, (io, size)), (L.tsr_linear_backward_bytes, (gr, size))):
        assert call(ctypes.byref(d), *[ctypes.byref(a) for a in args]) == status
    assert L.tsr_linear_forward(ctypes.byref(d), ctypes.byref(io), AT, 1 << 40, None) == status
    assert L.tsr_linear_backward(ctypes.byref(d), ctypes.byref(gr), AT, 1 << 40, None) == status


def test_linear_refuses_matrices_and_scratch(tsr):
    L, M = tsr.lib(), tsr.Matrix
    none, size = M(None, 0), ctypes.c_size_t()
    d = linear_desc(tsr)
    base = dict(x=M(AT, 8), weight=M(AT, 8), residual=none, pre=none, y=M(AT, 16), bias=None)

    def fwd(**kw):
        io = tsr.LinearIO(*dict(base, **kw).values())
        return L.tsr_linear_forward_bytes(ctypes.byref(d), ctypes.byref(io), ctypes.byref(size))

    assert fwd() == 0
    assert fwd(x=none) == 1 and fwd(weight=none) == 1 and fwd(y=none) == 1
    assert fwd(x=M(AT, 7)) == 2 and fwd(weight=M(AT, 7)) == 2 and fwd(y=M(AT, 15)) == 2 and fwd(residual=M(AT, 15)) == 2 and fwd(pre=M(AT, 15)) == 2
    assert fwd(x=M(AT + 1, 8)) == 3 and fwd(y=M(AT + 1, 16)) == 3 and fwd(bias=AT + 2) == 3
    assert L.tsr_linear_forward_bytes(None, None, ctypes.byref(size)) == 1 and L.tsr_linear_forward_bytes(ctypes.byref(d), None, None) == 1
    assert fwd(x=M(AT + 2, 8)) == 0 and size.value >= 100 * 8 * 2        # an operand that is copied needs scratch
    io = tsr.LinearIO(*dict(base, x=M(AT + 2, 8)).values())
    assert L.tsr_linear_forward(ctypes.byref(d), ctypes.byref(io), None, 0, None) == 4
    assert L.tsr_linear_forward(ctypes.byref(d), ctypes.byref(io), AT, size.value - 1, None) == 4
    assert L.tsr_linear_forward(ctypes.byref(d), ctypes.byref(io), AT + 128, size.value, None) == 3

    g = dict(dy=M(AT, 16), x=M(AT, 8), weight=M(AT, 8), pre=none, dx=M(AT, 8), dweight=M(AT, 8), dbias=None)

    def bwd(d=d, **kw):
        gr = tsr.LinearGrads(*dict(g, **kw).values())
        return L.tsr_linear_backward_bytes(ctypes.byref(d), ctypes.byref(gr), ctypes.byref(size))

    assert bwd() == 0
    assert bwd(dy=none) == 1 and bwd(x=none) == 1 and bwd(weight=none) == 1 and bwd(linear_desc(tsr, activation=2)) == 1
    assert bwd(x=none, dweight=none) == 0 and bwd(weight=none, dx=none) == 0
    assert bwd(dx=M(AT, 7)) == 2 and bwd(dweight=M(AT, 7)) == 2 and bwd(dweight=M(AT + 2, 8)) == 3 and bwd(dbias=AT + 2) == 3
    assert bwd(d=linear_desc(tsr, rows=1000), dbias=AT) == 0 and size.value > 0      # (few rows add their column sums within one cluster)


def test_dropout_refuses(tsr):
    L, M = tsr.lib(), tsr.Matrix
    ok, none = M(AT, 8), M(None, 0)

    def call(p=0.5, dtype=0, rows=4, cols=8, x=ok, r=none, y=ok):
        return L.tsr_dropout(ctypes.byref(tsr.DropoutDesc(p, 0, 0, 0, None)), dtype, rows, cols, x, r, y, None)

    assert call(p=-1.0) == 1 and call(p=float("nan")) == 1 and call(dtype=2) == 6 and call(rows=-1) == 2 and call(cols=1 << 31) == 2 and call(rows=(1 << 40) + 1) == 2
    assert call(x=none) == 1 and call(y=none) == 1 and call(x=M(AT, 7)) == 2 and call(r=M(AT, 7)) == 2 and call(y=M(AT + 1, 8)) == 3
    assert L.tsr_dropout(None, 0, 4, 8, ok, none, ok, None) == 1
    assert call(rows=0) == 0 and call(cols=0) == 0
    for p in (-0.1, 1.1, float("nan")):
        with pytest.raises(ValueError):
            tsr.Dropout(p, 0)
    with pytest.raises(ValueError):
        tsr.Dropout(0.1, 0, step=torch.zeros(1, dtype=torch.int64))


def test_tensors_on_the_host_are_refused(tsr):
    x, w = torch.zeros(3, 4), torch.zeros(5, 4)
    for call in (lambda: tsr.norm_forward(x), lambda: tsr.linear_forward(x, w), lambda: tsr.linear_backward(x, None, w.t()), lambda: tsr.dropout_forward(x, tsr.Dropout(0.1, 0)),
                 lambda: tsr.norm_backward(x, x, None, x), lambda: tsr.layer_norm(x), lambda: tsr.linear(x, w)):
        with pytest.raises(ValueError):
            call()


def test_layouts(tsr):
    from paper_2602_08007_b200.layers import _layout
    t = torch.zeros(6, 8, 10)
    assert _layout(t) == (48, 10, 10)
    assert _layout(t[:, :, :7]) == (48, 7, 10)
    assert _layout(t[:, ::2]) == (24, 10, 20)
    assert _layout(t[:, :5]) is None and _layout(t[::2]) is None          # two pitches
    assert _layout(t.transpose(1, 2)) is None and _layout(t[:, :, ::2]) is None
    assert _layout(t[0, 0]) == (1, 10, 10) and _layout(t[0, 0, ::3]) is None
    assert _layout(torch.zeros(1, 4).expand(5, 4)) is None                # rows that overlap
    assert _layout(torch.zeros(5, 1).expand(5, 4)) is None
    assert _layout(t[2:3, :, 1:4]) == (8, 3, 10) and _layout(t[:, 3:4, 1:4]) == (6, 3, 80)
    assert _layout(torch.zeros(())) is None
    assert _layout(torch.zeros(0, 5))[:2] == (0, 5) and _layout(torch.zeros(3, 0))[:2] == (3, 0) and _layout(torch.zeros(4, 3, 0))[:2] == (12, 0)
    assert _layout(torch.zeros(7, 9)[:, 2:3]) == (7, 1, 9)


def test_words_of_dropout():
    """The model's own words, against plain integers."""
    def mix(x):
        x &= 0xFFFFFFFF
        x ^= x >> 16
        x = x * 0x85EBCA6B & 0xFFFFFFFF
        x ^= x >> 13
        x = x * 0xC2B2AE35 & 0xFFFFFFFF
        return x ^ x >> 16

    seed, offset, p = (7 << 32) + 3, (5 << 32) + 9, 0.37
    k = mix(mix(seed ^ mix((seed >> 32) + 0x9E3779B9)) ^ mix(offset + 0x7F4A7C15))
    k = mix(k ^ ((offset >> 32) * 0x85EBCA77 & 0xFFFFFFFF))
    first = (3 << 32) - 2
    got = lm.kept(4, 7, p, seed, offset, first)
    for i in range(4):
        row = first + i
        r1 = mix(k ^ mix(row % 2 ** 32 + 0x9E3779B9 * ((row >> 32) + 1)))
        r2 = mix(r1 ^ 0xA511E9B3)
        for c in range(7):
            x = (c // 2 + r1) & 0xFFFFFFFF
            x ^= x >> 16
            x = x * 0x85EBCA6B & 0xFFFFFFFF
            x ^= x >> 13 ^ r2
            x = x * 0xC2B2AE35 & 0xFFFFFFFF
            x ^= x >> 16
            bits = x >> 16 if c & 1 else x & 0xFFFF
            assert got[i, c] == (bits >= int(np.floor(float(np.float32(p)) * 65536 + 0.5)))


def test_addresses_that_are_read_in_pairs(tsr):
    """(mu, r) and the dropout word are eight bytes each."""
    L, M = tsr.lib(), tsr.Matrix
    d, m, none = norm_desc(tsr), M(AT, 8), M(None, 0)
    assert L.tsr_norm_forward(ctypes.byref(d), m, None, None, m, AT + 4, None) == 3
    assert L.tsr_norm_backward(ctypes.byref(d), m, m, None, AT + 4, m, None, None, AT, 1 << 30, None) == 3
    drop = tsr.DropoutDesc(0.5, 0, 0, 0, AT + 4)
    assert L.tsr_dropout(ctypes.byref(drop), 0, 4, 8, m, none, m, None) == 1


def test_one_row_of_the_longest_length_is_split(tsr):
    """The kernel for few rows counts K in 32 bits; beyond its limit a product that splits K takes over, with scratch for the parts."""
    L, M = tsr.lib(), tsr.Matrix
    none, size = M(None, 0), ctypes.c_size_t()
    for K, scratch in ((1 << 24, False), ((1 << 24) + 8, True), (0x7fffffff - 1023, True)):
        d = tsr.LinearDesc(1, K, 8, 0, 0, 0, 0, 0, 0, tsr.DropoutDesc(0.0, 0, 0, 0, None))
        io = tsr.LinearIO(M(AT, K), M(AT, K), none, none, M(AT, 8), None)
        assert L.tsr_linear_forward_bytes(ctypes.byref(d), ctypes.byref(io), ctypes.byref(size)) == 0
        assert (size.value > 0) == scratch


def test_calls_by_keyword(tsr):
    """Every argument has a name, the one that says where to run too (CPU tensors get as far as the check)."""
    t = torch.zeros(4, 8)
    calls = [lambda: tsr.norm_forward(x=t, weight=None), lambda: tsr.norm_backward(dy=t, x=t, weight=None, stats=t), lambda: tsr.linear_forward(x=t, weight=t),
             lambda: tsr.linear_backward(dy=t, x=t, weight=t), lambda: tsr.dropout_forward(x=t, dropout=tsr.Dropout(0.1, 0)),
             lambda: tsr.dropout_backward(dy=t, dropout=tsr.Dropout(0.1, 0))]
    for call in calls:
        with pytest.raises(ValueError, match="CUDA device"):
            call()

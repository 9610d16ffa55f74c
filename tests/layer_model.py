"""The layer operators in 64 bits, from their formulas, and the bounds of what FP32 arithmetic and one rounding may add.

Roundings: half a step is 2^-8 of a BF16 value and 2^-24 of an FP32 one.  A tensor-core instruction adds the products of 16 BF16 (8 TF32)
pairs to the accumulator and keeps 24 bits of the largest term at least: it is off by at most 2^-22 of the sum of magnitudes."""

# FP32 products are six products of three BF16 parts of each operand, added within 128 entries of K by the tensor cores and in FP32 beyond.  The bound of
# product_slack below, that of two TF32 parts, is wider than what they keep; test_gpu_linear_f32.py checks each of the six and the size of the error.
# Activations go through the special-function units, in FP32 layers with corrections (test_gpu_layer_activations.py); the bounds below hold for both.
import math

import numpy as np
import torch

HALF = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}
ACTS = ["none", "relu", "gelu", "gelu_tanh", "silu"]


def close(got, want, slack):
    """Every entry within half a step of its own type and `slack`; what is not finite has to be the same."""
    assert got.shape == want.shape, (got.shape, want.shape)
    got64 = got.double()
    fine = torch.isfinite(want)
    assert torch.equal(torch.isnan(got64), torch.isnan(want)) and torch.equal(got64[~fine & ~torch.isnan(want)], want[~fine & ~torch.isnan(want)])
    off = (got64 - want).abs()
    bound = HALF[got.dtype] * (want.abs() + slack) + slack + 1e-38
    bad = fine & ~(off <= bound)
    assert not bad.any(), "%d of %d entries; worst %g at %s" % (int(bad.sum()), bad.numel(), float((off / bound)[fine].max()), bad.nonzero()[0].tolist())


def mix(a):
    a = a.astype(np.uint32).copy()
    a ^= a >> np.uint32(16)
    a *= np.uint32(0x85EBCA6B)
    a ^= a >> np.uint32(13)
    a *= np.uint32(0xC2B2AE35)
    return a ^ (a >> np.uint32(16))


def word32(v):
    return np.array([v % 2 ** 32], dtype=np.uint32)


def threshold(p):
    return int(math.floor(float(np.float32(p)) * 65536.0 + 0.5))


def kept(rows, cols, p, seed, offset, first_row=0):
    """Truth values: which entries of rows first_row ... dropout keeps."""
    k = mix(mix(word32(seed) ^ mix(word32((seed >> 32) + 0x9E3779B9))) ^ mix(word32(offset % 2 ** 32 + 0x7F4A7C15)))
    k = mix(k ^ word32((offset >> 32) * 0x85EBCA77))
    row = np.arange(first_row, first_row + rows, dtype=np.uint64)
    r1 = mix(k ^ mix(((row & 0xFFFFFFFF) + 0x9E3779B9 * ((row >> np.uint64(32)) + np.uint64(1))).astype(np.uint32)))
    r2 = mix(r1 ^ np.uint32(0xA511E9B3))
    x = np.arange((cols + 1) // 2, dtype=np.uint32)[None, :] + r1[:, None]
    x ^= x >> np.uint32(16)
    x *= np.uint32(0x85EBCA6B)
    x = x ^ (x >> np.uint32(13)) ^ r2[:, None]
    x *= np.uint32(0xC2B2AE35)
    x ^= x >> np.uint32(16)
    return np.stack([x & np.uint32(0xFFFF), x >> np.uint32(16)], axis=2).reshape(rows, -1)[:, :cols] >= threshold(p)


def drop(x, d):
    """Dropout of a float64 matrix; d: None or a library Dropout."""
    if d is None or threshold(d.p) == 0:
        return x
    t = threshold(d.p)
    off = (d.offset + (int(d.step) if d.step is not None else 0)) % 2 ** 64
    keep = torch.from_numpy(kept(x.shape[0], x.shape[1], d.p, d.seed, off)).to(x.device)
    return torch.where(keep, x * (65536.0 / (65536 - t) if t < 65536 else 0.0), torch.zeros((), dtype=x.dtype, device=x.device))


def factor(d):
    t = 0 if d is None else threshold(d.p)
    return 0.0 if t == 65536 else 65536.0 / (65536 - t)


def act(kind, z):
    if kind == "relu":
        return z.clamp(min=0.0)
    if kind == "gelu":
        return z * 0.5 * torch.special.erfc(-z * math.sqrt(0.5))
    if kind == "gelu_tanh":
        return z * torch.sigmoid(2.0 * math.sqrt(2.0 / math.pi) * (z + 0.044715 * z ** 3))
    if kind == "silu":
        return z * torch.sigmoid(z)
    return z


def slope(kind, z):
    if kind == "relu":
        return (z > 0).double()
    if kind == "gelu":
        return 0.5 * torch.special.erfc(-z * math.sqrt(0.5)) + z * torch.exp(-0.5 * z * z) / math.sqrt(2.0 * math.pi)
    if kind == "gelu_tanh":
        k = 2.0 * math.sqrt(2.0 / math.pi)
        s = torch.sigmoid(k * (z + 0.044715 * z ** 3))
        return s + z * s * (1.0 - s) * k * (1.0 + 3.0 * 0.044715 * z ** 2)
    if kind == "silu":
        s = torch.sigmoid(z)
        return s + z * s * (1.0 - s)
    return torch.ones_like(z)


def product_slack(a, b, dtype):
    """Bound on a b^T formed from operands of `dtype` (float64 tensors): accumulation, and for FP32 the split of the operands (2^-22 of each, and
    the product of the low parts)."""
    s = a.abs() @ b.abs().t()
    steps = a.shape[1] / 16 + 2 if dtype == torch.bfloat16 else 3 * a.shape[1] / 8 + 2 + 3
    return s * (steps * 2.0 ** -22)


def linear(x, w, bias=None, kind="none", drop_=None, residual=None):
    """(y, pre, slack of y, slack of pre) in 64 bits for inputs as they are."""
    dt = x.dtype
    x, w = x.double(), w.double()
    z = x @ w.t()
    sz = product_slack(x, w, dt)
    if bias is not None:
        z = z + bias.double()
        sz = sz + 2.0 ** -23 * z.abs()
    a = act(kind, z)
    # slopes stay below 1.2; expf, erff and the quotient are within 2^-20 of the values they meet (|z| + 1)
    sy = sz if kind == "none" else 1.2 * sz + 2.0 ** -20 * (z.abs() + 1.0)
    y = drop(a, drop_)
    sy = sy * max(1.0, factor(drop_)) + 2.0 ** -23 * y.abs()
    if residual is not None:
        y = y + residual.double()
        sy = sy + 2.0 ** -23 * (y.abs() + residual.double().abs())
    return y, z, sy, sz


def linear_grads(dy, x, w, pre=None, kind="none", drop_=None):
    """((dx, slack), (dw, slack), (db, slack)) in 64 bits."""
    dt = dy.dtype
    dy, x, w = dy.double(), x.double(), w.double()
    dz = dy
    sdz = torch.zeros_like(dz)
    if kind != "none":
        z = pre.double()
        dz = dz * slope(kind, z)
        sdz = 2.0 ** -19 * dy.abs() * (z.abs() + 1.0)
    dz = drop(dz, drop_)
    if drop_ is not None:
        sdz = sdz * factor(drop_) + 2.0 ** -22 * dz.abs()
    rounded = HALF[dt] * dz.abs() if kind != "none" or drop_ is not None else torch.zeros_like(dz)
    op = sdz + rounded
    dx = dz @ w, op @ w.abs() + product_slack(dz.abs() + op, w.t(), dt)
    dw = dz.t() @ x, op.t() @ x.abs() + product_slack((dz.abs() + op).t(), x.t(), dt)
    # column sums: at most 2^9 additions one after the other on any path
    db = dz.sum(0), sdz.sum(0) + 2.0 ** -15 * dz.abs().sum(0)
    return dx, dw, db


def norm(x, w=None, b=None, eps=1e-5, center=True):
    """(y, slack, mean, slack, rstd, slack) in 64 bits.  A sum has at most 2^7 additions on any path: 2^-17 of the magnitudes."""
    x = x.double()
    n = x.shape[1]
    mu = x.mean(1, keepdim=True) if center else torch.zeros(x.shape[0], 1, dtype=torch.float64, device=x.device)
    smu = 2.0 ** -17 * x.abs().mean(1, keepdim=True) if center else torch.zeros_like(mu)
    d = x - mu
    q = (d * d).sum(1, keepdim=True) / n
    rstd = 1.0 / torch.sqrt(q + float(np.float32(eps)))
    # the distance is off by smu and a rounding each, which moves q by twice that times |d|, and by the square
    sd = smu + 2.0 ** -23 * (x.abs() + mu.abs())
    sq = 2.0 ** -17 * q + 2.0 * (d.abs() * sd).mean(1, keepdim=True) + (sd * sd).mean(1, keepdim=True)
    srstd = rstd * (0.5 * sq / (q + float(np.float32(eps))) + 2.0 ** -22)
    h = d * rstd
    wv = torch.ones(n, dtype=torch.float64, device=x.device) if w is None else w.double()
    bv = torch.zeros(n, dtype=torch.float64, device=x.device) if b is None else b.double()
    y = h * wv + bv
    sy = wv.abs() * (sd * rstd + d.abs() * srstd) + 2.0 ** -22 * (h.abs() * wv.abs() + bv.abs())
    return y, sy, mu, smu, rstd, srstd


def norm_grads(dy, x, w, stats, center=True):
    """((dx, slack), (dw, slack), (db, slack)) in 64 bits for the given statistics."""
    dy, x = dy.double(), x.double()
    mu, rs = stats[:, :1].double(), stats[:, 1:].double()
    wv = torch.ones(x.shape[1], dtype=torch.float64, device=x.device) if w is None else w.double()
    h = (x - mu) * rs
    sh = 2.0 ** -22 * (x.abs() + mu.abs()) * rs
    g = dy * wv
    c1 = g.mean(1, keepdim=True) if center else torch.zeros_like(mu)
    c2 = (g * h).mean(1, keepdim=True)
    s1 = 2.0 ** -17 * g.abs().mean(1, keepdim=True)
    s2 = 2.0 ** -17 * (g * h).abs().mean(1, keepdim=True) + (g.abs() * sh).mean(1, keepdim=True)
    dx = rs * (g - c1 - h * c2)
    sdx = rs * (s1 + h.abs() * s2 + sh * c2.abs() + 2.0 ** -21 * (g.abs() + c1.abs() + (h * c2).abs()))
    dw = (dy * h).sum(0)
    sdw = 2.0 ** -15 * (dy * h).abs().sum(0) + (dy.abs() * sh).sum(0)
    db = dy.sum(0)
    return (dx, sdx), (dw, sdw), (db, 2.0 ** -15 * dy.abs().sum(0))

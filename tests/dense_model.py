"""Plain models of the dense-parameter operators for the tests: the definition in 64 bits (numpy), and the stored bits of
the 8-bit state from IEEE FP32 operations (numpy float32).  They share no code with the library."""
import math

import numpy as np
import torch

U24 = 2.0 ** -24          # relative error of one FP32 rounding
BLOCK = 256


def f32(x):
    return float(np.float32(x))


def to64(t):
    return t.detach().cpu().to(torch.float64).numpy()


# E4M3: values of all 256 codes, from sign, exponent and mantissa
def _e4m3_value(c):
    s, e, m = c >> 7, (c >> 3) & 15, c & 7
    if e == 15 and m == 7:
        return math.nan
    x = m * 2.0 ** -9 if e == 0 else (1 + m / 8) * 2.0 ** (e - 7)
    return -x if s else x


E4M3 = np.array([_e4m3_value(c) for c in range(256)])
POSITIVE = E4M3[:127]     # ascending


def spacing(y):
    """Distance of neighbouring E4M3 values around |y| <= 448."""
    with np.errstate(divide="ignore"):
        return 2.0 ** (np.maximum(np.floor(np.log2(np.abs(y))), -6.0) - 3.0)


def bf16_unit(x):
    """Distance of neighbouring BF16 values (8 significant bits) at |x|."""
    with np.errstate(divide="ignore"):
        return 2.0 ** (np.maximum(np.floor(np.log2(np.abs(x))), -126.0) - 7.0)


def blocks(x, fill=0.0):
    """A flat array as rows of 256, padded with `fill`."""
    n = len(x)
    out = np.full(((n + BLOCK - 1) // BLOCK, BLOCK), fill, dtype=x.dtype)
    out.reshape(-1)[:n] = x
    return out


def step64(p, g, m, v, h, s=1.0, lr_mult=1.0, wd_mult=1.0):
    """One AdamW step in 64 bits and, element by element, how far FP32 arithmetic may be from it: one U24 for every
    rounding that the FP32 form makes (two for an approximate square root, four for an approximate quotient).
    Returns (p, m, v, tol_p, tol_m, tol_v); h: dict of lr, beta1, beta2, eps, wd, t (FP32 values)."""
    b1, b2, t = h["beta1"], h["beta2"], h["t"]
    lr, wd = h["lr"] * lr_mult, h["wd"] * wd_mult
    g = g * s
    m1 = b1 * m + (1 - b1) * g
    v1 = b2 * v + (1 - b2) * g * g
    den = np.sqrt(v1 / (1 - b2 ** t)) + h["eps"]
    d = m1 / (1 - b1 ** t) / den
    p1 = (1 - lr * wd) * p - lr * d
    tol_m = 4 * U24 * (np.abs(b1 * m) + np.abs((1 - b1) * g)) + 1e-44
    tol_v = 7 * U24 * v1 + 1e-44
    tol_d = 16 * U24 * np.abs(d) + tol_m / (1 - b1 ** t) / den
    tol_p = 4 * U24 * np.abs(p) + U24 * np.abs(p1) + lr * tol_d
    return p1, m1, v1, tol_p, tol_m, tol_v


def random_words(counter, k1, k2):
    x = counter.astype(np.uint32) + np.uint32(k1)
    x ^= x >> np.uint32(16)
    x *= np.uint32(0x85EBCA6B)
    x = x ^ (x >> np.uint32(13)) ^ np.uint32(k2)
    x *= np.uint32(0xC2B2AE35)
    return x ^ (x >> np.uint32(16))


def mix32(x):
    x &= 0xFFFFFFFF
    x ^= x >> 16
    x = x * 0x85EBCA6B & 0xFFFFFFFF
    x ^= x >> 13
    x = x * 0xC2B2AE35 & 0xFFFFFFFF
    return x ^ (x >> 16)


def keys(seed, step, tensor):
    a = mix32((seed & 0xFFFFFFFF) ^ mix32((seed >> 32) + 0x9E3779B9))
    k1 = mix32(a ^ mix32((step & 0xFFFFFFFF) + 0x7F4A7C15 * (tensor + 1)))
    return k1, mix32(k1 ^ 0xA511E9B3)


def scale_of(x):
    """Per row of x >= 0 (float32): the smallest power of two >= 2^-126 with max x <= 448 * scale, by trial."""
    out = np.empty((x.shape[0], 1))
    for i, a in enumerate(x.max(axis=1).astype(np.float64)):
        if not np.isfinite(a):
            out[i] = np.nan
            continue
        e = -126
        while a > 448.0 * 2.0 ** e:
            e += 1
        out[i] = 2.0 ** e
    return out


def quantise(x, scale, bits16=None):
    """E4M3 codes of x / scale (float64 arithmetic on float32 values, so exact): nearest, ties to the even code, or up in
    magnitude where the 16 random bits exceed the remainder."""
    y = np.abs(x.astype(np.float64)) / scale
    y = np.where(np.isfinite(y), y, 0.0)
    lo = np.clip(np.searchsorted(POSITIVE, y, side="right") - 1, 0, 125)
    below, above = POSITIVE[lo], POSITIVE[lo + 1]
    if bits16 is None:
        up = (y - below > above - y) | ((y - below == above - y) & (lo % 2 == 1))
    else:
        # the FP32 word of y (of y + 2^-6 below 2^-6, rounded to FP32) has 20 bits under the mantissa's first three; the
        # random bits are added 4 bits up, and a carry moves to the next value
        small = y < 2.0 ** -6
        z = np.where(small, y + 2.0 ** -6, y).astype(np.float32).astype(np.float64)
        base = np.where(small, below + 2.0 ** -6, below)
        unit = np.where(small, 2.0 ** -9, above - below)
        base = np.where(small & (z >= above + 2.0 ** -6), above + 2.0 ** -6, base)
        lo = np.where(small & (z >= above + 2.0 ** -6), lo + 1, lo)
        rest = np.floor((z - base) / unit * 2.0 ** 20 + 0.5).astype(np.int64)
        up = rest + (bits16.astype(np.int64) << 4) >= 2 ** 20
    code = np.where(up, lo + 1, lo)
    return np.where(np.signbit(x), code | 128, code).astype(np.uint8)


def step_bits(g, cm, cr, scale, h, s=None, rkeys=None):
    """The 8-bit state after one step, bit for bit, from IEEE FP32 operations.  g: float32, flat; cm, cr: codes (uint8, flat);
    scale: (blocks, 2) float32.  Returns (codes of m, codes of r, scales, m, r) with m, r the new FP32 moments."""
    F = np.float32
    n = len(g)
    if s is not None:
        g = g * F(s)
    sm, sr = (np.repeat(scale[:, k], BLOCK)[:n] for k in (0, 1))
    m = E4M3[cm].astype(F) * sm
    r = E4M3[cr].astype(F) * sr
    omb1, omb2 = F(1.0 - h["beta1"]), F(1.0 - h["beta2"])
    with np.errstate(all="ignore"):
        m1 = F(h["beta1"]) * m + omb1 * g
        r1 = np.sqrt(F(h["beta2"]) * (r * r) + omb2 * (g * g))
    bm, br = blocks(m1), blocks(r1)
    s1 = np.concatenate([scale_of(np.abs(bm)), scale_of(br)], axis=1)
    bits = None
    if rkeys is not None:
        w = random_words(np.arange(bm.size, dtype=np.uint32), *rkeys).reshape(bm.shape)
        bits = (w & np.uint32(0xFFFF), w >> np.uint32(16))
    c1 = quantise(bm, s1[:, :1], bits and bits[0])
    c2 = quantise(br, s1[:, 1:], bits and bits[1])
    c2 = np.where((br > 0) & (c2 == 0), 1, c2).astype(np.uint8)
    return c1.reshape(-1)[:n], c2.reshape(-1)[:n], s1.astype(F), m1, r1

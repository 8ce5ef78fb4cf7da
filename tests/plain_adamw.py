"""One AdamW step over one tensor on the host, as include/zq.h defines it: in binary32
operations one after another (the bits a kernel has to give), and in binary64 with the
distance that binary32 roundings may put between the two."""
import math

import numpy as np

F = np.float32


def e4m3(code):
    """Values of e4m3 codes (bias 7): by the definition of the format."""
    code = np.asarray(code, np.int64)
    e, m = code >> 3 & 15, code & 7
    v = np.where(e == 0, m / 8.0 * 2.0**-6, (1 + m / 8.0) * 2.0 ** (e - 7.0))
    return np.where(code & 128, -v, v)


def e5m2(code):
    code = np.asarray(code, np.int64)
    e, m = code >> 2 & 31, code & 3
    return np.where(e == 0, m / 4.0 * 2.0**-14, (1 + m / 4.0) * 2.0 ** (e - 15.0))


def mix(x):
    x = np.asarray(x, np.uint64) & np.uint64(0xFFFFFFFF)
    low = np.uint64(0xFFFFFFFF)
    x = x ^ (x >> np.uint64(16))
    x = x * np.uint64(0x6A09E667) & low
    x = x ^ (x >> np.uint64(15))
    x = x * np.uint64(0x3B67AE85) & low
    return x ^ (x >> np.uint64(16))


def drawn(step, tensor, first, n):
    """32 bits for elements first .. first + n - 1 (within one 2^32 of them)."""
    key = int(mix(int(mix(step)) + tensor * 0x9E3779B9))
    if first >> 32:
        key = int(mix(key + (first >> 32)))
    return mix(np.arange(first & 0xFFFFFFFF, (first & 0xFFFFFFFF) + n, dtype=np.uint64) ^ np.uint64(key))


def blocks(x, block):
    return np.pad(x, (0, -len(x) % block)).reshape(-1, block)


def spread(scales, block, n):
    return np.repeat(scales, block)[:n]


def encode8(x, bits16, block, signed):
    """codes and scales of binary32 x: each value on the grid of the codes, up with the
    chance of what is cut off (16 bits of it)."""
    top, value, last = (448.0, e4m3, 126) if signed else (57344.0, e5m2, 123)
    a = blocks(np.abs(x), block).max(1)
    fits = a >= F(2.0**-110)
    safe = np.where(fits, a, F(1))
    scales = np.where(fits, a / F(top), F(0)).astype(F)
    r = np.where(fits, F(top) / safe, F(0)).astype(F)
    y = (np.abs(x) * spread(r, block, len(x))).astype(F).astype(np.float64)
    grid = value(np.arange(last + 1))
    at = np.clip(np.searchsorted(grid, y, side="right") - 1, 0, last)
    up = np.minimum(at + 1, last)
    width = np.where(up > at, grid[up] - grid[at], 1.0)
    # the part above the code, in as many bits as binary32 (or the code grid's lowest
    # step) has below a code's, and the drawn half-open sixteenth bits
    cut = 20 if signed else 21
    unit = 2.0 ** (-126.0 + 120.0 - 23.0) if signed else 2.0 ** (-126.0 + 112.0 - 23.0)
    exponent = np.maximum(np.frexp(np.maximum(y, 1e-300))[1] - 1, -6 if signed else -14)
    lsb = 2.0 ** (exponent - 23.0)
    assert (lsb >= unit).all()
    part = np.rint((y - grid[at]) / lsb)  # y is a multiple of lsb but below the grid's normal range, where it is rounded to one
    assert (part <= 2.0**cut).all() and (width / lsb <= 2.0**cut).all()
    bump = bits16.astype(np.float64) * 2.0 ** (cut - 16) + 2.0 ** (cut - 17)
    code = np.where(part + bump >= 2.0**cut, at + 1, at)
    code = np.minimum(code, last)
    return (code + (128 * (x < 0) if signed else 0)).astype(np.uint8), scales


def decode8(codes, scales, block, signed):
    return ((e4m3 if signed else e5m2)(codes).astype(F) * spread(scales, block, len(codes))).astype(F)


def clip_factor(scale, norm, max_norm):
    if norm is None:
        return F(scale)
    ratio = F(max_norm) / F(F(norm) + F(1e-6))
    return F(F(scale) * (F(1) if ratio > 1 else ratio))


def step32(p, g, m, v, t, lr, b1, b2, eps, wd, lr_scale=1.0):
    """(p before its cast, m, v) in binary32, from binary32 arrays; g already clipped."""
    root = F(1.0 / math.sqrt(1.0 - b2**t))
    rate = lr * lr_scale
    alpha, decay = F(rate / (1.0 - b1**t)), F(1.0 - rate * wd)
    m = m * F(b1) + g * F(1.0 - b1)
    v = v * F(b2) + (g * g) * F(1.0 - b2)
    return p * decay - (m / (np.sqrt(v) * root + F(eps))) * alpha, m, v


def step64(p, g, m, v, t, lr, b1, b2, eps, wd, lr_scale=1.0):
    """The same in binary64, and the bounds of what binary32 may differ by.  A rounding is
    2^-24 of its value.  m: two constants, two products, g's three (its factor's two, the
    product) and a sum: 8 of the terms' magnitudes.  v: g's three twice, its square, a
    constant, a product, the other term's two, a sum: 10.  The update: m's error over d, half of
    v's 10, root's two, the product, the sum with eps (and eps), the quotient, alpha's
    two: 14 of it.  p: its decay's two, and the difference."""
    p, g, m, v = (np.asarray(x, np.float64) for x in (p, g, m, v))
    u = 2.0**-24
    rate = lr * lr_scale
    m1, v1 = b1 * m + (1 - b1) * g, b2 * v + (1 - b2) * g * g
    d = np.sqrt(v1 / (1 - b2**t)) + eps
    alpha = rate / (1 - b1**t)
    step = alpha * m1 / d
    m_off = 8 * u * (np.abs(b1 * m) + np.abs((1 - b1) * g))
    new = p * (1 - rate * wd) - step
    return (new, m1, v1), (u * (3 * np.abs(p) + 14 * np.abs(step) + np.abs(new)) + np.abs(alpha) * m_off / d, m_off,
                           10 * u * v1)

"""The AdamW step and its states in 8 bits, written out in numpy: in 64 bits, and operation by operation in fp32 (which says every code)."""
from __future__ import annotations

import numpy as np

GOLDEN, MASK = 0x9E3779B97F4A7C15, (1 << 64) - 1
F = np.float32


def output(z):
    z = np.asarray(z, dtype=np.uint64)
    with np.errstate(over="ignore"):
        z = (z ^ (z >> np.uint64(30))) * np.uint64(0xBF58476D1CE4E5B9)
        z = (z ^ (z >> np.uint64(27))) * np.uint64(0x94D049BB133111EB)
    return z ^ (z >> np.uint64(31))


def draws(seed, t, tensor, n):
    key = int(output((int(output((seed + t * GOLDEN) & MASK)) + (tensor + 1) * GOLDEN) & MASK))
    with np.errstate(over="ignore"):
        w = output(np.uint64(key) + (np.arange((n + 1) // 2, dtype=np.uint64) + np.uint64(1)) * np.uint64(GOLDEN))
    half = np.stack([w & np.uint64(0xFFFFFFFF), w >> np.uint64(32)], 1).reshape(-1)[:n].astype(np.uint32)
    return half & 0xFFFF, half >> 16


def blocks(x):
    return np.pad(x, (0, -len(x) % 32)).reshape(-1, 32)


def encode(x, u, positive):
    """codes and bytes of fp32 values, a 16-bit draw each"""
    n = len(x)
    with np.errstate(all="ignore"):
        b = blocks(x.astype(F))
        a = np.abs(b)
        bits = a.view(np.uint32).max(1)  # infinities and NaNs above every number
        e = np.maximum((bits >> 23).astype(np.int64) - 135 + ((bits & 0x7FFFFF) > 0x600000), -117)
        ok = bits < 0x7F000000
        e = np.where(ok, e, 0)
        y = a * np.ldexp(F(1), -e).astype(F)[:, None]
        binade = np.maximum((y.view(np.uint32) >> 23).astype(np.int64), 121)
        up = blocks(u.astype(F)) * F(2.0 ** -16)
        step = np.ldexp(F(1), 130 - np.minimum(binade, 200)).astype(F)
        code = (binade - 121) * 8 + np.floor((y * step).astype(F) + up).astype(np.int64)
        if positive:
            code = np.where(a > 0, np.maximum(code, 1), code)
        else:
            code = code + 128 * np.signbit(b)
    code[~ok] = 0x7F
    return code.reshape(-1)[:n].astype(np.uint8), np.where(ok, e + 127, 255).astype(np.uint8)


def decode(code, scale):
    """fp64 numbers (exact)"""
    c = blocks(code.astype(np.int64))
    size, sign = c & 127, np.where(c & 128, -1.0, 1.0)
    value = np.where(size < 8, size * 2.0 ** -9, (8 + size % 8) * 2.0 ** (size // 8 - 10.0))
    value = np.where(size == 127, np.nan, value)
    s = scale.astype(np.int64)[:, None]
    factor = np.where(s == 0, 0.0, np.where(s == 255, np.inf, 2.0 ** (s - 127.0)))
    with np.errstate(invalid="ignore"):
        return (sign * value * factor).reshape(-1)[:len(code)]


def step_64(p, g, m, v, lr, b1, b2, eps, wd, t, scale=1.0):
    """v: the mean of squares.  All in fp64, the rates as fp32 holds them."""
    lr, b1, b2, eps, wd, scale = (float(F(x)) for x in (lr, b1, b2, eps, wd, scale))
    p, g, m, v = (np.asarray(x, dtype=np.float64) for x in (p, g, m, v))
    g = g * scale
    m = b1 * m + (1 - b1) * g
    v = b2 * v + (1 - b2) * g * g
    return p * (1 - lr * wd) - lr * (m / (1 - b1 ** t)) / (np.sqrt(v / (1 - b2 ** t)) + eps), m, v


def means_32(g, m, v, b1, b2, scale=1.0):
    """m and the root of v as every operation in fp32 gives them (v: fp32)."""
    g, m, v, b1, b2 = F(scale) * g.astype(F), m.astype(F), v.astype(F), F(b1), F(b2)
    with np.errstate(all="ignore"):
        return b1 * m + (F(1) - b1) * g, np.sqrt(b2 * v + (F(1) - b2) * g * g)

"""Rows held in 8 bits, written from the format's definition in float64 (test infrastructure): codes e4m3, a power of two per 128 channels."""
import math

import numpy as np

MOST, LEAST = 448.0, -126
MAG = np.array([c / 512.0 if c < 8 else 2.0 ** (c // 8 - 7) * (1 + c % 8 / 8.0) for c in range(127)])
EDGES = (MAG[1:] + MAG[:-1]) / 2


def lds(C):
    return -(-C // 128) * 128, -(-C // 512) * 4


def scale_exponent(top):
    """The smallest e >= -126 with top <= 448 * 2^e."""
    if top == 0:
        return LEAST
    e = max(LEAST, math.ceil(math.log2(top / MOST)) - 1)
    while MOST * 2.0 ** e < top:
        e += 1
    return e


def nearest_code(a):
    """Codes of the magnitudes nearest to a >= 0 (ties to the even code)."""
    c = np.searchsorted(EDGES, a)
    edge = (c < 126) & (a == EDGES[np.minimum(c, 125)]) & (c % 2 == 1)
    return (c + edge).astype(np.uint8)


def store(x):
    """[rows, C] float64 -> (codes, scales) as sige_rows8_store leaves them; NaN codes where x is not finite (their sign bit 0)."""
    rows, C = x.shape
    ld, sld = lds(C)
    q, s = np.zeros((rows, ld), np.uint8), np.zeros((rows, sld), np.uint8)
    for b in range(-(-C // 128)):
        g = x[:, 128 * b:min(C, 128 * b + 128)]
        fine = np.isfinite(g)
        for r in range(rows):
            e = scale_exponent(np.abs(np.where(fine[r], g[r], 0.0)).max())
            s[r, b] = e + 127
            a = np.where(fine[r], np.abs(g[r]), 0.0) * 2.0 ** -e
            q[r, 128 * b:128 * b + g.shape[1]] = np.where(fine[r], nearest_code(a) | np.where(np.signbit(g[r]), 0x80, 0).astype(np.uint8), 0x7f)
    return q, s


def values(q, s, C):
    """What codes and scales stand for."""
    c = q[:, :C].astype(int)
    v = np.where(c & 127 == 127, np.nan, MAG[np.minimum(c & 127, 126)]) * np.where(c > 127, -1.0, 1.0)
    e = np.repeat(s[:, :-(-C // 128)].astype(float), 128, 1)[:, :C]
    return v * np.where(e == 255, np.nan, 2.0 ** (e - 127))


def gate(g, kind):
    """gelu (0) or silu (1)."""
    erfc = np.vectorize(math.erfc, otypes=[float])
    return g * 0.5 * erfc(-g / math.sqrt(2.0)) if kind == 0 else g / (1.0 + np.exp(-np.clip(g, -700, None)))

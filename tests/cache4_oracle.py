"""The cache of keys and values in 4 bits, in float64 NumPy from its definition: quantisation, byte layout, the attention that
reads it.  Test infrastructure only."""
import numpy as np
import torch

GRID = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
E_RANGE = {torch.float32: (-125, 125), torch.bfloat16: (-125, 125), torch.float16: (-23, 13)}


def sections(d):
    """(planes of 32 channels, planes of 16, scale bytes per token)"""
    g = -(-d // 32)
    tail = int(0 < d % 32 <= 16)
    return g - tail, tail, next(n for n in (1, 2, 4, 8) if n >= g)


def quantise(x, dtype):
    """[..., d] float64 -> codes 0..15 [..., 32 * groups], scale bytes [..., groups]; a group that is not finite: codes 0, byte 255."""
    lo, hi = E_RANGE[dtype]
    d = x.shape[-1]
    groups = -(-d // 32)
    g = np.zeros(x.shape[:-1] + (groups * 32,))
    g[..., :d] = x
    g = g.reshape(x.shape[:-1] + (groups, 32))
    finite = np.isfinite(g).all(-1)
    g = np.where(finite[..., None], g, 0.0)
    top = np.abs(g).max(-1)
    e = np.full(top.shape, lo)
    for _ in range(lo, hi):                    # the smallest exponent that holds the largest value
        e = np.where(top > 6 * 2.0 ** e, e + 1, e)
    a = np.abs(g) / 2.0 ** e[..., None]
    code = np.zeros(a.shape, int)
    for i in range(1, 8):
        border = (GRID[i - 1] + GRID[i]) / 2
        code = np.where((a > border) | ((a == border) & (i % 2 == 0)), i, code)
    code = code + 8 * (g < 0)
    return code.reshape(x.shape[:-1] + (groups * 32,)), np.where(finite, e + 127, 255)


def values(code, byte, last=252):
    """float64 values of codes and scale bytes (NaN beyond `last`)."""
    v = GRID[code & 7] * np.where(code & 8, -1.0, 1.0)
    s = np.where(byte > last, np.nan, 2.0 ** (byte.astype(float) - 127))
    return v * np.repeat(s, 32, -1)


def views(cache, heads, d, capacity):
    """Per head and (keys, values): writable views (planes [F][cap][16], short plane [cap][8] or None, scales [cap][gs])."""
    full, tail, gs = sections(d)
    cap = -(-capacity // 32) * 32
    sec = cache.reshape(heads, 2, cap * (16 * full + 8 * tail + gs))
    out = []
    for h in range(heads):
        row = []
        for w in range(2):
            s = sec[h, w]
            a, b = full * cap * 16, full * cap * 16 + tail * cap * 8
            row.append((s[:a].reshape(full, cap, 16), s[a:b].reshape(cap, 8) if tail else None, s[b:].reshape(cap, gs)))
        out.append(row)
    return out


def put(cache, heads, d, capacity, token, code, byte, which):
    """Writes codes [heads][32 G] and bytes [heads][G] of one token into the byte array."""
    full, tail, _ = sections(d)
    v = views(cache, heads, d, capacity)
    for h in range(heads):
        planes, short, scales = v[h][which]
        pair = (code[h, 0::2] | code[h, 1::2] << 4).astype(np.uint8)
        for g in range(full):
            planes[g, token] = pair[16 * g:16 * g + 16]
        if tail:
            short[token] = pair[16 * full:16 * full + 8]
        scales[token, :full + tail] = byte[h]


def read(cache, heads, d, capacity, T, which, last=252):
    """[T, heads, d] float64 values of the first T tokens."""
    full, tail, _ = sections(d)
    v = views(cache, heads, d, capacity)
    out = np.zeros((T, heads, 32 * (full + tail)))
    for h in range(heads):
        planes, short, scales = v[h][which]
        code = np.zeros((T, 32 * (full + tail)), int)
        for g in range(full):
            code[:, 32 * g:32 * g + 32:2] = planes[g, :T] & 15
            code[:, 32 * g + 1:32 * g + 32:2] = planes[g, :T] >> 4
        if tail:
            code[:, 32 * full:32 * full + 16:2] = short[:T] & 15
            code[:, 32 * full + 1:32 * full + 16:2] = short[:T] >> 4
        out[:, h] = values(code, scales[:T, :full + tail], last)
    return out[:, :, :d]


def attention(q, k, v, scale, ranges=None):
    """o [Nq, heads, d] and sum_t (p_t + 2^-30) |v_t|; a row that sees nothing is zero, what a row does not see does not reach it."""
    nq, heads, d = q.shape
    T = k.shape[0]
    o, mag = np.zeros((nq, heads, d)), np.zeros((nq, heads, d))
    groups = {}
    for i in range(nq):
        b, e = (0, T) if ranges is None else (max(int(ranges[i][0]), 0), min(int(ranges[i][1]), T))
        groups.setdefault((b, e), []).append(i)
    for (b, e), rows in groups.items():
        if b >= e:
            continue
        for h in range(heads):
            s = q[rows, h] @ k[b:e, h].T * scale
            with np.errstate(invalid="ignore"):
                p = np.exp(s - s.max(1, keepdims=True))
                p /= p.sum(1, keepdims=True)
                o[rows, h] = p @ v[b:e, h]
                mag[rows, h] = (p + 2.0 ** -30) @ np.abs(v[b:e, h])
    return o, mag

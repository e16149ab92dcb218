"""Rotary positions with several axes on the GPU against their definition in float64."""
import math

import numpy as np
import pytest
import torch

from paper_2211_02048_amd import api

pytestmark = pytest.mark.gpu
DT = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
# sine and cosine and the angle's own rounding; half types take the hardware's sines, single precision the library's
SIN = {"f32": 2.0 ** -22, "f16": 2.0 ** -18, "bf16": 2.0 ** -18}


def f64(t):
    return t.detach().cpu().double().numpy()


def turns_of(axis_pairs, theta):
    f = np.concatenate([theta ** (-np.arange(p) / max(p, 1)) for p in axis_pairs])
    return f, np.concatenate([np.full(p, a) for a, p in enumerate(axis_pairs)]).astype(int)


def rotate(x, pos, axis_pairs, theta, layout):
    """x [rows, heads, d] float64, pos [rows, axes]; also |a| + |b| of each value's pair."""
    f, axis = turns_of(axis_pairs, theta)
    n = len(f)
    t = pos[:, axis] * f
    y, mag = x.copy(), np.zeros_like(x)
    ia, ib = (np.arange(n), np.arange(n) + n) if layout else (2 * np.arange(n), 2 * np.arange(n) + 1)
    a, b = x[:, :, ia], x[:, :, ib]
    c, s = np.cos(t)[:, None], np.sin(t)[:, None]
    y[:, :, ia], y[:, :, ib] = a * c - b * s, a * s + b * c
    mag[:, :, ia] = mag[:, :, ib] = np.abs(a) + np.abs(b)
    return y, mag


def check(y, x, pos, axis_pairs, theta, layout, heads, d, dtype):
    want, mag = rotate(f64(x).reshape(-1, heads, d), pos, axis_pairs, theta, layout)
    # the sines' error and two fp32 roundings on |a| + |b|, the rounding of the result
    bound = mag * (SIN[dtype] + 2.0 ** -23) + torch.finfo(DT[dtype]).eps / 2 * np.abs(want)
    got = f64(y).reshape(want.shape)
    assert (np.abs(got - want) <= bound).all(), np.max(np.abs(got - want) / np.maximum(bound, 1e-30))
    flat = mag == 0
    assert np.array_equal(got[flat], f64(x).reshape(want.shape)[flat])


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("layout", [api.ROPE_ADJACENT, api.ROPE_HALVES])
@pytest.mark.parametrize("rows,heads,d,axis_pairs", [
    (1, 1, 8, (4,)), (3, 2, 40, (10, 10)), (77, 5, 72, (12, 12, 12)), (33, 3, 80, (13, 20)), (130, 16, 64, (8, 12, 12)),
    (9, 2, 24, (3, 2)), (5, 1, 256, (64, 0, 64)), (2000, 1, 16, (1,)), (11, 7, 128, (3, 3, 3, 3)),
])
def test_positions(rows, heads, d, axis_pairs, layout, dtype):
    rng = np.random.default_rng(rows + d)
    td = DT[dtype]
    wide = torch.from_numpy(rng.standard_normal((rows, heads * d + 24))).to(td).cuda()
    x = wide[:, 8:8 + heads * d]
    pos = rng.integers(-5, 100, (rows, len(axis_pairs))).astype(np.float32)
    pos[0] = 1e6 + 1                              # far: the angle's whole turns are taken off exactly
    pos[-1] = 0.5
    table = api.sige_rope_pairs(axis_pairs, 10000.0)
    p = torch.from_numpy(pos).cuda()
    out = torch.full((rows + 1, heads * d + 8), 7.0, dtype=td, device="cuda")
    api.sige_token_rope(x, out[:rows, :heads * d], heads, d, table, p, layout=layout, n_rows=rows)
    torch.cuda.synchronize()
    check(out[:rows, :heads * d], x, pos.astype(np.float64), axis_pairs, 10000.0, layout, heads, d, dtype)
    assert (out[rows] == 7.0).all() and (out[:, heads * d:] == 7.0).all()
    before = wide.clone()                         # in place
    api.sige_token_rope(x, x, heads, d, table, p, layout=layout, n_rows=rows)
    torch.cuda.synchronize()
    assert torch.equal(x, out[:rows, :heads * d])
    assert torch.equal(wide[:, :8], before[:, :8]) and torch.equal(wide[:, 8 + heads * d:], before[:, 8 + heads * d:])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("axes", [2, 3])
def test_positions_by_block_list(axes, dtype):
    """The positions of the listed blocks' pixels; the count on the host and on the device, rows past it left as they were."""
    heads, d, b, side, frame = 4, 40, 4, 18, 11.0
    g = api.geom(side, side, b, 1, 1, 0)
    blocks = np.array([[0, 0], [4, 8], [16, 16]], np.int32)
    n, cap = 3, 5
    idx = torch.zeros((cap, 2), dtype=torch.int32)
    idx[:n] = torch.from_numpy(blocks)
    x = torch.randn(cap * b * b, heads * d, dtype=torch.float64).to(DT[dtype]).cuda()
    yx = np.array([[y0 + p // b, x0 + p % b] for y0, x0 in blocks for p in range(b * b)], float)
    pos = yx if axes == 2 else np.concatenate([np.full((len(yx), 1), frame), yx], 1)
    pairs = (10, 10) if axes == 2 else (4, 8, 8)
    table = api.sige_rope_pairs(pairs, 100.0)
    for n_blocks in (n, -1):
        y = torch.full_like(x, 7.0)
        api.sige_token_rope_blocks(x, y, heads, d, table, g, idx.cuda(), torch.tensor([n], dtype=torch.int32, device="cuda"),
                                   n_axes=axes, frame=frame, n_blocks=n_blocks)
        torch.cuda.synchronize()
        check(y[:n * b * b], x[:n * b * b], pos, pairs, 100.0, 0, heads, d, dtype)
        assert (y[n * b * b:] == 7.0).all()


def test_device_count_and_axes_that_are_not_there():
    heads, d, rows = 2, 16, 40
    x = torch.randn(rows, heads * d, device="cuda")
    table = api.sige_rope_pairs((4, 4), 50.0)
    table[5, 2] = 2                               # no positions for this axis, nor for that one
    table[6, 2] = -1
    pos = torch.randint(0, 50, (rows, 2), device="cuda").float()
    y = torch.full_like(x, 7.0)
    api.sige_token_rope(x, y, heads, d, table, pos, count=torch.tensor([3], dtype=torch.int32, device="cuda"), rows_per_count=9)
    torch.cuda.synchronize()
    assert (y[27:] == 7.0).all()
    p = f64(pos)[:27]
    want, mag = rotate(f64(x)[:27].reshape(27, heads, d), p, (4, 4), 50.0, 0)
    got = f64(y)[:27].reshape(27, heads, d)
    x64 = f64(x)[:27].reshape(27, heads, d)
    want[:, :, 10:14] = x64[:, :, 10:14]
    assert (np.abs(got - want) <= mag * (2.0 ** -22 + 2.0 ** -23) + 2.0 ** -24 * np.abs(want)).all()


def test_rotation_is_undone_by_the_opposite_positions():
    """Turning by -p after p gives the rows back (the operator's transpose, hence its gradient, is itself at -p)."""
    heads, d, rows = 3, 64, 50
    x = torch.randn(rows, heads * d, device="cuda")
    table = api.sige_rope_pairs((16, 16))
    pos = torch.rand(rows, 2, device="cuda") * 1000
    y, z = torch.empty_like(x), torch.empty_like(x)
    api.sige_token_rope(x, y, heads, d, table, pos, n_rows=rows)
    api.sige_token_rope(y, z, heads, d, table, -pos, n_rows=rows)
    torch.cuda.synchronize()
    # twice the error of one turn, on |a| + |b| <= 2 max
    assert float((z - x).abs().max()) <= 4 * float(x.abs().max()) * (2.0 ** -22 + 2.0 ** -22)
    assert math.isclose(float((y * y).sum()), float((x * x).sum()), rel_tol=1e-4)

"""Rows in 8 bits on the GPU against their definitions in float64: store, load, the root-mean-square norm, the product and its gated form."""
import numpy as np
import pytest
import torch

import rows8_oracle as ref
from paper_2211_02048_amd import api

pytestmark = pytest.mark.gpu
DT = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
TINY = {"f32": 2.0 ** -150, "f16": 2.0 ** -25, "bf16": 2.0 ** -134}     # half a step of the type's smallest numbers


def f64(t):
    return t.detach().cpu().double().numpy()


def rounded(a, dtype):
    return torch.from_numpy(np.ascontiguousarray(a)).to(DT[dtype]).double().numpy()


def rows(seed, n, C, dtype, extra=8):
    """Rows of a wider tensor, channels of unlike size."""
    g = torch.Generator().manual_seed(seed)
    x = torch.full((n, C + extra), 3.0, dtype=torch.float64)
    x[:, :C] = torch.randn(n, C, generator=g, dtype=torch.float64) * torch.exp(torch.randn(C, generator=g, dtype=torch.float64))
    return x.to(DT[dtype]).cuda()[:, :C]


def room(n, C, more=1, wide=16):
    """Codes and scales with a row and bytes behind, all 0xa5."""
    ld, sld = ref.lds(C)
    return (torch.full((n + more, ld + wide), 0xa5, dtype=torch.uint8, device="cuda"), torch.full((n + more, sld + 4), 0xa5, dtype=torch.uint8, device="cuda"))


def check_room(q, s, n, C):
    """Nothing behind the rows or their bytes was written; codes and scale bytes behind C are 0."""
    ld, sld = ref.lds(C)
    assert (q[n:] == 0xa5).all() and (s[n:] == 0xa5).all() and (q[:, ld:] == 0xa5).all() and (s[:, sld:] == 0xa5).all()
    assert (q[:n, C:ld] == 0).all() and (s[:n, -(-C // 128):sld] == 0).all()


def same_codes(q, s, x64, C):
    wq, ws = ref.store(x64)
    gq, gs = q.cpu().numpy()[:, :wq.shape[1]], s.cpu().numpy()[:, :ws.shape[1]]
    np.testing.assert_array_equal(gs, ws)
    nan = wq & 0x7f == 0x7f
    np.testing.assert_array_equal(gq[~nan], wq[~nan])
    assert (gq[nan] & 0x7f == 0x7f).all()


# ---- store, load ---------------------------------------------------------------------------------------

@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("n,C", [(1, 8), (1, 128), (3, 136), (17, 320), (640, 40), (5, 512), (33, 520), (7, 1288), (4, 8192), (2, 16384)])
def test_store_and_load(n, C, dtype):
    x = rows(n + C, n, C, dtype)
    q, s = room(n, C)
    api.sige_rows8_store(x, q, s, C, n_rows=n)
    torch.cuda.synchronize()
    same_codes(q[:n], s[:n], f64(x), C)
    check_room(q, s, n, C)
    for out in ("bf16", "f16", "f32"):
        y = torch.full((n + 1, C + 8), 7.0, dtype=DT[out], device="cuda")
        api.sige_rows8_load(q, s, y[:n, :C], C, n_rows=n)
        torch.cuda.synchronize()
        np.testing.assert_array_equal(f64(y[:n, :C]), rounded(ref.values(q[:n].cpu().numpy(), s[:n].cpu().numpy(), C), out))
        assert (y[n] == 7.0).all() and (y[:, C:] == 7.0).all()


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
def test_store_borders(dtype):
    """Every code and every tie at several scales, maxima at and beside 448 times a power of two, zeros, subnormal numbers, the type's ends."""
    cases = []
    for e in (-3, 0, 5):
        v = np.concatenate([ref.MAG, ref.EDGES])
        for part in np.array_split(np.concatenate([v, -v]), 5):
            cases.append(np.concatenate([part, [448.0]]) * 2.0 ** (e if dtype != "f16" else min(e, 3)))
    end = float(torch.finfo(DT[dtype]).max)
    least = float(torch.finfo(DT[dtype]).smallest_normal)
    for top in (448.0, 449.0, 450.0, 447.0, 480.0, 1.75, 1.7578125, 1.75 * 2.0 ** -10, end, least, least / 4, 0.0, least * 448, least * 450):
        cases.append(np.array([top, -top / 2, top / 3, 0.0, -0.0, top / 1000]))
    x = np.zeros((len(cases), 128))
    for r, c in enumerate(cases):
        x[r, :len(c)] = c
    t = torch.from_numpy(x).to(DT[dtype]).cuda()
    q, s = room(len(cases), 128)
    api.sige_rows8_store(t, q, s, 128, n_rows=len(cases))
    torch.cuda.synchronize()
    same_codes(q[:-1], s[:-1], f64(t), 128)


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
def test_store_of_what_is_not_finite(dtype):
    """Infinities and NaN become NaN by themselves; a block of nothing else has the smallest scale."""
    x = rows(3, 6, 264, dtype, 0).clone()
    x[0, 5], x[1, 200], x[2, 130] = float("inf"), float("-inf"), float("nan")
    x[3, 128:256] = float("nan")
    x[4] = float("inf")
    q, s = room(6, 264)
    api.sige_rows8_store(x, q, s, 264, n_rows=6)
    y = torch.empty(6, 264, dtype=DT[dtype], device="cuda")
    api.sige_rows8_load(q, s, y, 264, n_rows=6)
    torch.cuda.synchronize()
    same_codes(q[:6], s[:6], f64(x), 264)
    assert torch.equal(torch.isnan(y), ~torch.isfinite(x))
    s[5, 0] = 255                                  # a block whose scale is NaN
    api.sige_rows8_load(q, s, y, 264, n_rows=6)
    torch.cuda.synchronize()
    assert torch.isnan(y[5, :128]).all() and torch.isfinite(y[5, 128:]).all()


def test_rows_by_a_count_on_the_device():
    n, C = 40, 320
    x = rows(1, n, C, "bf16")
    for count, per in ((3, 7), (0, 7), (9, 5), (-4, 7)):
        have = max(0, min(count * per, n))
        q, s = room(n, C)
        kw = dict(count=torch.tensor([count], dtype=torch.int32, device="cuda"), rows_per_count=per, max_rows=n)
        api.sige_rows8_store(x, q, s, C, **kw)
        y, z = (torch.full((n, C), 7.0, dtype=torch.bfloat16, device="cuda") for _ in range(2))
        api.sige_rows8_load(q, s, y, C, **kw)
        o, os_ = room(n, C)
        api.sige_token_rms(x, C, y=z, q=o, scales=os_, **kw)
        torch.cuda.synchronize()
        check_room(q, s, have, C)
        check_room(o, os_, have, C)
        assert (y[have:] == 7.0).all() and (z[have:] == 7.0).all()
        if have:
            same_codes(q[:have], s[:have], f64(x[:have]), C)
            np.testing.assert_array_equal(f64(y[:have]), ref.values(q[:have].cpu().numpy(), s[:have].cpu().numpy(), C))
            assert (z[:have] != 7.0).any(1).all()


# ---- norm ----------------------------------------------------------------------------------------------

def rms_expected(x, res, gamma, eps, dtype):
    h = f64(x)
    if res is not None:
        # (the sum is added in fp32 and rounded: two roundings, the second of a value that the first has moved by 2^-24 of itself)
        h = rounded(rounded(h + f64(res), "f32"), dtype)
    n = h / np.sqrt((h * h).mean(1, keepdims=True) + eps)
    return h, n if gamma is None else n * f64(gamma)


def close_codes(q, s, want, err, C, what=""):
    """8-bit rows of values that are off by at most err from `want`: half a step of e4m3 (2^-4 of the value, 2^-10 of the scale, or of
    twice the scale where the block's maximum lies beside a border)."""
    n = want.shape[0]
    got = ref.values(q[:n].cpu().numpy(), s[:n].cpu().numpy(), C)
    top = np.zeros((n, -(-C // 128)))
    for b in range(top.shape[1]):
        top[:, b] = (np.abs(want) + err)[:, 128 * b:128 * b + 128].max(1)
    scale = 2.0 ** np.vectorize(ref.scale_exponent)(top).astype(float)
    scale = np.repeat(scale, 128, 1)[:, :C]
    bound = err + 2.0 ** -4 * (np.abs(want) + err) + 2.0 ** -10 * scale
    off = np.abs(got - want)
    assert (off <= bound).all(), f"{what}: {np.nanmax(off / bound):.2f} of the bound"
    # the scale byte itself: that of the largest value, or its neighbour where err reaches the border
    low = np.zeros_like(top)
    for b in range(top.shape[1]):
        low[:, b] = np.maximum(np.abs(want) - err, 0)[:, 128 * b:128 * b + 128].max(1)
    e = s[:n, :top.shape[1]].cpu().numpy().astype(int) - 127
    assert (e <= np.vectorize(ref.scale_exponent)(top)).all() and (e >= np.vectorize(ref.scale_exponent)(low)).all(), what


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("n,C", [(1, 8), (5, 128), (3, 136), (19, 320), (6, 512), (7, 640), (5, 1288), (9, 2048), (3, 2056), (1, 4096), (4, 5120), (2, 8192), (2100, 640), (2060, 1032)])
def test_rms(n, C, dtype):
    x, res = rows(C + n, n, C, dtype), rows(C + n + 1, n, C, dtype, 16)
    gamma = (torch.rand(C + 3, dtype=torch.float32) + 0.5).cuda()[3:] if C % 16 else (torch.rand(C) + 0.5).cuda()     # (also not 16-byte aligned)
    for r, gm, eps in ((res, gamma, 1e-6), (None, gamma, 1e-5), (res, None, 0.0)):
        h, want = rms_expected(x, r, gm, eps, dtype)
        rel = (C / 2 + 16) * 2.0 ** -24         # the sum of C squares in fp32 under a root; division, root, two products
        y = torch.full((n + 1, C + 8), 7.0, dtype=DT[dtype], device="cuda")
        total = torch.full((n + 1, C + 8), 7.0, dtype=DT[dtype], device="cuda")
        q, s = room(n, C)
        api.sige_token_rms(x, C, gm, eps, residual=r, total=None if r is None else total[:n, :C], y=y[:n, :C], q=q, scales=s, n_rows=n)
        torch.cuda.synchronize()
        err = np.abs(f64(y[:n, :C]) - want)
        bound = rel * np.abs(want) + torch.finfo(DT[dtype]).eps / 2 * (1 + rel) * np.abs(want) + TINY[dtype]
        assert (err <= bound).all(), np.max(err / bound)
        close_codes(q, s, want, rel * np.abs(want), C, "norm")
        check_room(q, s, n, C)
        assert (y[n] == 7.0).all() and (y[:, C:] == 7.0).all() and (total[n] == 7.0).all() and (total[:, C:] == 7.0).all()
        if r is None:
            assert (total == 7.0).all()
        else:
            np.testing.assert_array_equal(f64(total[:n, :C]), h)
        # one output at a time: the same bits; in place
        y2, (q2, s2) = torch.empty_like(x), room(n, C)
        api.sige_token_rms(x, C, gm, eps, residual=r, q=q2, scales=s2, n_rows=n)
        api.sige_token_rms(x, C, gm, eps, residual=r, y=y2, n_rows=n)
        z = x.clone()
        api.sige_token_rms(z, C, gm, eps, residual=r, y=z, n_rows=n)
        torch.cuda.synchronize()
        assert torch.equal(y2, y[:n, :C]) and torch.equal(z, y2) and torch.equal(q, q2) and torch.equal(s, s2)
        if r is not None:
            z, w = x.clone(), r.clone()
            api.sige_token_rms(z, C, gm, eps, residual=w, total=w, y=z, n_rows=n)
            torch.cuda.synchronize()
            assert torch.equal(z, y2) and torch.equal(w, total[:n, :C])


def test_rms_widest_rows():
    for dtype, C in (("bf16", 16384), ("f16", 12296), ("f32", 8192), ("f32", 6148)):
        x = rows(C, 3, C, dtype)
        _, want = rms_expected(x, None, None, 1e-6, dtype)
        y, (q, s) = torch.empty_like(x), room(3, C)
        api.sige_token_rms(x, C, None, 1e-6, y=y, q=q, scales=s, n_rows=3)
        torch.cuda.synchronize()
        rel = (C / 2 + 16) * 2.0 ** -24
        assert (np.abs(f64(y) - want) <= (rel + torch.finfo(DT[dtype]).eps / 2 * (1 + rel)) * np.abs(want) + TINY[dtype]).all()
        close_codes(q, s, want, rel * np.abs(want), C)
        check_room(q, s, 3, C)


@pytest.mark.parametrize("C", [320, 4096])
def test_rms_rows_that_are_not_finite(C):
    """A NaN makes its row NaN, an infinity its row 0 and itself NaN; a row of zeros stays zeros; neighbours do not notice."""
    x = rows(2, 6, C, "bf16").clone()
    x[1, 7], x[2, 9], x[3] = float("nan"), float("inf"), 0.0
    y, (q, s) = torch.empty_like(x), room(6, C)
    api.sige_token_rms(x, C, None, 1e-6, y=y, q=q, scales=s, n_rows=6)
    back = torch.empty_like(x)
    api.sige_rows8_load(q, s, back, C, n_rows=6)
    torch.cuda.synchronize()
    for t in (y, back):
        assert torch.isnan(t[1]).all() and torch.isnan(t[2, 9]) and (torch.cat([t[2, :9], t[2, 10:]]) == 0).all() and (t[3] == 0).all()
        assert torch.isfinite(t[[0, 4, 5]]).all()
    want = rms_expected(x[[0, 4, 5]], None, None, 1e-6, "bf16")[1]
    assert (np.abs(f64(y[[0, 4, 5]]) - want) <= 2.0 ** -7.9 * np.abs(want)).all()


# ---- products ------------------------------------------------------------------------------------------

def matrix(seed, n, C, size=1.0, wide=0):
    """A matrix in 8 bits and its values; scales of unlike size from block to block."""
    rng = np.random.default_rng(seed)
    x = rng.normal(size=(n, C)) * np.exp(0.7 * rng.normal(size=C)) * 2.0 ** rng.integers(-2, 3, (n, 1)) * size
    q, s = ref.store(x)
    return wide_codes(q, s, wide) + (ref.values(q, s, C),)


def wide_codes(q, s, wide):
    a = torch.full((q.shape[0], q.shape[1] + wide), 0x7f, dtype=torch.uint8)       # what lies behind the codes is never read: NaN
    b = torch.full((s.shape[0], s.shape[1] + wide // 4), 0xff, dtype=torch.uint8)
    a[:, :q.shape[1]], b[:, :s.shape[1]] = torch.from_numpy(q), torch.from_numpy(s)
    return a.cuda(), b.cuda()


def product(xv, wv, cin):
    """The product, the sum of the magnitudes and what the 8-bit instruction may cut off: per product less than 2^-13 of the largest of its block."""
    y, mag = xv @ wv.T, np.abs(xv) @ np.abs(wv).T
    cut = np.zeros_like(y)
    for b in range(0, cin, 128):
        p, w = np.abs(xv[:, b:b + 128]), np.abs(wv[:, b:b + 128])
        for i in range(len(p)):
            cut[i] += p.shape[1] * 2.0 ** -13 * (p[i] * w).max(1)
    return y, mag, cut


SIZES = [(1, 8, 8), (1, 320, 960), (16, 1280, 136), (17, 128, 24), (5, 136, 16), (33, 640, 320), (64, 384, 256), (100, 520, 264), (257, 264, 72), (130, 1288, 144), (300, 1024, 520),
         (31, 2560, 640)]


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("n,cin,cout", SIZES)
def test_linear(n, cin, cout, dtype):
    xq, xs, xv = matrix(n + cin, n, cin, wide=16)
    wq, ws, wv = matrix(cout + cin, cout, cin, cin ** -0.5, wide=32)
    rng = np.random.default_rng(5)
    bias = torch.from_numpy(rng.normal(size=cout)).float().cuda()
    base = torch.from_numpy(rng.normal(size=(n, cout + 8))).to(DT[dtype]).cuda()[:, :cout]
    want, mag, cut = product(xv, wv, cin)
    for b, r in ((bias, base), (None, None), (None, base)):
        y = torch.full((n + 1, cout + 8), 7.0, dtype=DT[dtype], device="cuda")
        api.sige_rows8_linear(xq, xs, wq, ws, y[:n, :cout], cin, cout, bias=b, base=r, n_rows=n)
        torch.cuda.synchronize()
        more = (0 if b is None else f64(b)) + (0 if r is None else f64(r))
        w = want + more
        bound = (cin + 4) * 2.0 ** -24 * (mag + np.abs(more)) + (0 if dtype == "f32" else cut)
        bound = bound + torch.finfo(DT[dtype]).eps / 2 * (np.abs(w) + bound) + TINY[dtype]
        err = np.abs(f64(y[:n, :cout]) - w)
        assert (err <= bound).all(), f"{np.max(err / bound):.2f} of the bound"
        assert (y[n] == 7.0).all() and (y[:, cout:] == 7.0).all()
    z = base.clone()
    api.sige_rows8_linear(xq, xs, wq, ws, z, cin, cout, base=z, n_rows=n)
    torch.cuda.synchronize()
    assert torch.equal(z, y[:n, :cout])


@pytest.mark.parametrize("gate", [api.GATE_GELU, api.GATE_SILU])
@pytest.mark.parametrize("n,cin,cout", SIZES)
def test_gated(n, cin, cout, gate):
    xq, xs, xv = matrix(n + cin, n, cin, wide=16)
    wq, ws, wv = matrix(cout + cin, 2 * cout, cin, 0.5 * cin ** -0.5, wide=32)
    bias = torch.from_numpy(np.random.default_rng(5).normal(size=2 * cout)).float().cuda()
    want, mag, cut = product(xv, wv, cin)
    for b in (bias, None):
        more = 0 if b is None else f64(b)
        err = (cin + 4) * 2.0 ** -24 * (mag + np.abs(more)) + cut
        u, g = (want + more)[:, :cout], (want + more)[:, cout:]
        v = u * ref.gate(g, gate)
        # the sums' errors (the gates' slope is below 1.13), then the gate's own: its polynomial is off by 2^-19.6, at most, of |g| / 2, some roundings
        off = err[:, :cout] * (np.abs(ref.gate(g, gate)) + 1.13 * err[:, cout:]) + np.abs(u) * 1.13 * err[:, cout:] + 2.0 ** -18 * np.abs(u * g)
        q, s = room(n, cout)
        api.sige_rows8_linear_gated(xq, xs, wq, ws, q, s, cin, cout, gate=gate, bias=b, n_rows=n)
        torch.cuda.synchronize()
        close_codes(q, s, v, off, cout, "gated")
        check_room(q, s, n, cout)


def on_gpu(q, s, C):
    """What codes and scales stand for, in float64 on the GPU."""
    c = q[:, :C].int()
    e, m = c >> 3 & 15, c & 7
    v = torch.where(e == 0, m / 512.0, torch.exp2(e.double() - 7) * (1 + m / 8.0)).double()
    k = torch.arange(C, device="cuda") // 128
    return torch.where(c > 127, -v, v) * torch.exp2(s[:, k].double() - 127)


def drawn(seed, n, C, size=1.0):
    """A matrix in 8 bits of normal numbers, made on the GPU."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn(n, C, generator=g, device="cuda") * torch.exp2(torch.randint(-2, 3, (n, 1), generator=g, device="cuda").float()) * size
    q, s = api.rows8(n, C)
    api.sige_rows8_store(x, q, s, C, n_rows=n)
    return q, s


def cut_of(xv, wv):
    """What the 8-bit instruction may cut off, bounded by the rows' largest values of each block (product() has it by the products)."""
    n, cin = xv.shape
    pad = -cin % 128
    top = lambda v: torch.nn.functional.pad(v.abs(), (0, pad)).unflatten(1, (-1, 128)).amax(-1)    # noqa: E731
    return 128 * 2.0 ** -13 * (top(xv) @ top(wv).t())


# rows, input and output channels: tiles that are not whole, one block and many, more tiles than compute units (the last round in halves)
FORM_SIZES = [(1, 128, 8), (70, 136, 72), (64, 640, 128), (129, 1288, 264), (200, 256, 520), (257, 1152, 256), (33, 3080, 40), (400, 384, 1032), (300, 8200, 136)]


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("form", range(8))
def test_forms_of_the_product(form, dtype):
    """Every kernel on every size, with a device count too, bit for bit the same from run to run."""
    if form == 7 and dtype == "f32":
        return
    sizes = FORM_SIZES + ([(4200, 136, 4104)] if form == 7 else []) + ([(37, 200, 12), (150, 264, 268)] if dtype == "f32" else [])
    sizes += [(2100, 264, 2200)] if form == 6 else []          # (workgroups that go from tile to tile, of which some are not whole)
    for n, cin, cout in sizes:
        x, w = drawn(n, n, cin), drawn(cout, cout, cin, cin ** -0.5)
        bias, base = torch.randn(cout, device="cuda"), torch.randn(n, cout, device="cuda").to(DT[dtype])
        xv, wv = on_gpu(*x, cin), on_gpu(*w, cin)
        want = xv @ wv.t() + bias.double() + base.double()
        bound = (cin + 4) * 2.0 ** -24 * (xv.abs() @ wv.abs().t() + bias.double().abs() + base.double().abs()) + (0 if dtype == "f32" else cut_of(xv, wv))
        bound = bound + torch.finfo(DT[dtype]).eps / 2 * (want.abs() + bound) + TINY[dtype]
        y = torch.full((n + 1, cout + 8), 7.0, dtype=DT[dtype], device="cuda")
        z, have = torch.full((n, cout), 7.0, dtype=DT[dtype], device="cuda"), min(n, 3 * (n // 5 + 1))
        with api.knobs(ROWS8_FORM=form):
            api.sige_rows8_linear(*x, *w, y[:n, :cout], cin, cout, bias=bias, base=base, n_rows=n)
            api.sige_rows8_linear(*x, *w, z, cin, cout, bias=bias, base=base, count=torch.tensor([3], dtype=torch.int32, device="cuda"), rows_per_count=n // 5 + 1, max_rows=n)
        torch.cuda.synchronize()
        off = (y[:n, :cout].double() - want).abs()
        assert (off <= bound).all(), (n, cin, cout, float((off / bound).max()))
        assert (y[n] == 7.0).all() and (y[:, cout:] == 7.0).all()
        assert torch.equal(z[:have], y[:have, :cout]) and (z[have:] == 7.0).all()


@pytest.mark.parametrize("gate", [api.GATE_GELU, api.GATE_SILU])
@pytest.mark.parametrize("form", range(4))
def test_forms_of_the_gated_product(form, gate):
    for n, cin, cout in FORM_SIZES + ([(2200, 136, 4104)] if form == 3 else [(1100, 520, 4104)] if form in (1, 2) else []):
        x, w = drawn(n, n, cin), drawn(cout, 2 * cout, cin, 0.5 * cin ** -0.5)
        bias = torch.randn(2 * cout, device="cuda")
        xv, wv = on_gpu(*x, cin), on_gpu(*w, cin)
        want = xv @ wv.t() + bias.double()
        err = (cin + 4) * 2.0 ** -24 * (xv.abs() @ wv.abs().t() + bias.double().abs()) + cut_of(xv, wv)
        u, g, eu, eg = want[:, :cout], want[:, cout:], err[:, :cout], err[:, cout:]
        act = g * torch.special.ndtr(g) if gate == api.GATE_GELU else g * torch.sigmoid(g)
        off = eu * (act.abs() + 1.13 * eg) + u.abs() * 1.13 * eg + 2.0 ** -18 * (u * g).abs()
        q, s = room(n, cout)
        o, os_ = room(n, cout)
        have = min(n, 3 * (n // 5 + 1))
        with api.knobs(ROWS8_FORM=form):
            api.sige_rows8_linear_gated(*x, *w, q, s, cin, cout, gate=gate, bias=bias, n_rows=n)
            api.sige_rows8_linear_gated(*x, *w, o, os_, cin, cout, gate=gate, bias=bias, count=torch.tensor([3], dtype=torch.int32, device="cuda"), rows_per_count=n // 5 + 1, max_rows=n)
        torch.cuda.synchronize()
        check_room(q, s, n, cout)
        check_room(o, os_, have, cout)
        assert torch.equal(o[:have], q[:have]) and torch.equal(os_[:have], s[:have])
        rows_ = range(n) if n <= 400 else list(range(0, n, 37)) + [n - 1]
        pick = torch.tensor(list(rows_), device="cuda")
        close_codes(q[pick], s[pick], f64((u * act)[pick]), f64(off[pick]), cout, (n, cin, cout))


def test_single_precision_loses_nothing():
    """Numbers whose products lie far apart, with a sum that cancels the large ones: the 8-bit instruction would cut the small ones off."""
    cin, n, cout = 256, 20, 24
    rng = np.random.default_rng(0)
    x, w = np.zeros((n, cin)), np.zeros((cout, cin))
    x[:, :64], w[:, :64] = 448.0, 448.0
    w[:, 32:64] = -448.0
    x[:, 64:128], w[:, 64:128] = rng.integers(1, 16, (n, 64)) / 64.0, rng.integers(1, 16, (cout, 64)) / 64.0
    (xq, xs), (wq, ws) = (wide_codes(*ref.store(v), 0) for v in (x, w))
    y = torch.empty(n, cout, device="cuda")
    api.sige_rows8_linear(xq, xs, wq, ws, y, cin, cout, n_rows=n)
    torch.cuda.synchronize()
    # partial sums of 32 products of 2^17.6 have 24 bits: 2^-1.4 each
    assert (np.abs(f64(y) - x @ w.T) <= cin * 2.0 ** -24 * 32 * 448.0 ** 2).all()
    x[:, :64] = 0
    xq, xs = wide_codes(*ref.store(x), 0)
    api.sige_rows8_linear(xq, xs, wq, ws, y, cin, cout, n_rows=n)
    torch.cuda.synchronize()
    np.testing.assert_array_equal(f64(y), x @ w.T)     # 64 products of 8 bits: exact


@pytest.mark.parametrize("form", [-1] + list(range(8)))
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_products_with_what_is_not_finite(dtype, form):
    """NaN codes and NaN scales reach the rows and channels that read them and no others."""
    if form == 7 and dtype == "f32":
        return
    n, cin, cout = 37, 392, 136
    xq, xs, _ = matrix(1, n, cin)
    wq, ws, _ = matrix(2, 2 * cout, cin)
    xq[3, 100] = 0x7f
    xs[20, 2] = 255
    wq[50, 391] = 0xff
    ws[77, 0] = 255
    y = torch.empty(n, cout, dtype=DT[dtype], device="cuda")
    q, s = room(n, cout)
    with api.knobs(ROWS8_FORM=form):
        api.sige_rows8_linear(xq, xs, wq, ws, y, cin, cout, n_rows=n)
    with api.knobs(ROWS8_FORM=min(form, 3)):
        api.sige_rows8_linear_gated(xq, xs, wq, ws, q, s, cin, cout, n_rows=n)
    back = torch.empty(n, cout, device="cuda")
    api.sige_rows8_load(q, s, back, cout, n_rows=n)
    torch.cuda.synchronize()
    for t in (y, back):
        bad = torch.zeros(n, cout, dtype=torch.bool, device="cuda")
        bad[[3, 20]], bad[:, [50, 77]] = True, True
        assert torch.equal(torch.isnan(t), bad)


@pytest.mark.parametrize("form", range(4))
def test_gated_values_that_overflow(form):
    """A gated value beyond fp32 becomes NaN by itself; its block's scale is that of the others."""
    n, cin, cout = 70, 128, 136
    x, w = np.ones((n, cin)), np.zeros((2 * cout, cin))
    w[:cout, 0], w[cout:, 0] = np.linspace(1.0, 2.0, cout), 3.0
    w[5], w[cout + 5] = 2.0 ** 100, 2.0 ** 60
    (xq, xs), (wq, ws) = (wide_codes(*ref.store(v), 0) for v in (x, w))
    q, s = room(n, cout)
    with api.knobs(ROWS8_FORM=form):
        api.sige_rows8_linear_gated(xq, xs, wq, ws, q, s, cin, cout, gate=api.GATE_SILU, n_rows=n)
    torch.cuda.synchronize()
    wv = ref.values(wq.cpu().numpy(), ws.cpu().numpy(), cin)[:, 0]
    v = wv[:cout] * ref.gate(wv[cout:], 1)
    got = ref.values(q[:n].cpu().numpy(), s[:n].cpu().numpy(), cout)
    rest = np.arange(cout) != 5
    assert np.isnan(got[:, 5]).all() and (s[:n, 0].cpu().numpy() == ref.scale_exponent(v[rest][:127].max()) + 127).all()
    assert (np.abs(got[:, rest] - v[rest]) <= (2.0 ** -4 + 2.0 ** -18) * v[rest]).all()


def test_extreme_scales():
    """Scales from one end to the other: sums beyond fp16 become infinite, tiny ones keep their bits in single precision."""
    n, cin, cout = 16, 256, 16
    for ex, ew in ((60, 40), (-60, -40), (100, -100), (-100, 100), (-55, -55)):
        rng = np.random.default_rng(1)
        x, w = rng.normal(size=(n, cin)) * 2.0 ** ex, rng.normal(size=(cout, cin)) * 2.0 ** ew
        (xq, xs), (wq, ws) = (wide_codes(*ref.store(v), 0) for v in (x, w))
        xv, wv = ref.values(xq.cpu().numpy(), xs.cpu().numpy(), cin), ref.values(wq.cpu().numpy(), ws.cpu().numpy(), cin)
        want, mag, cut = product(xv, wv, cin)
        for dtype in ("f32", "bf16"):
            y = torch.empty(n, cout, dtype=DT[dtype], device="cuda")
            api.sige_rows8_linear(xq, xs, wq, ws, y, cin, cout, n_rows=n)
            torch.cuda.synchronize()
            bound = (cin + 4) * 2.0 ** -24 * mag + (0 if dtype == "f32" else cut)
            bound = bound + torch.finfo(DT[dtype]).eps / 2 * (np.abs(want) + bound)
            assert (np.abs(f64(y) - want) <= bound + 2.0 ** -126).all(), (ex, ew, dtype)
    big = wide_codes(*ref.store(np.full((n, cin), 1000.0)), 0)
    y = torch.empty(n, cout, dtype=torch.float16, device="cuda")
    api.sige_rows8_linear(*big, *(t[:cout] for t in big), y, cin, cout, n_rows=n)
    torch.cuda.synchronize()
    assert torch.isinf(y).all()


def test_product_rows_by_a_count_on_the_device():
    n, cin, cout = 200, 264, 136
    xq, xs, xv = matrix(1, n, cin)
    wq, ws, wv = matrix(2, 2 * cout, cin)
    full = torch.empty(n, cout, device="cuda")
    api.sige_rows8_linear(xq, xs, wq, ws, full, cin, cout, n_rows=n)
    fq, fs = room(n, cout)
    api.sige_rows8_linear_gated(xq, xs, wq, ws, fq, fs, cin, cout, n_rows=n)
    for count, per in ((3, 16), (0, 16), (100, 16), (-1, 16), (1, 1), (5, 29)):
        have = max(0, min(count * per, n))
        kw = dict(count=torch.tensor([count], dtype=torch.int32, device="cuda"), rows_per_count=per, max_rows=n)
        y, (q, s) = torch.full((n, cout), 7.0, device="cuda"), room(n, cout)
        api.sige_rows8_linear(xq, xs, wq, ws, y, cin, cout, **kw)
        api.sige_rows8_linear_gated(xq, xs, wq, ws, q, s, cin, cout, **kw)
        torch.cuda.synchronize()
        assert torch.equal(y[:have], full[:have]) and (y[have:] == 7.0).all()
        assert torch.equal(q[:have], fq[:have]) and torch.equal(s[:have], fs[:have])
        check_room(q, s, have, cout)


def test_count_far_below_zero():
    """-10^9 * 4 is 294967296 in 32 bits, and no rows all the same: nothing is written."""
    n, C, cout = 200, 264, 136
    kw = dict(count=torch.tensor([-10 ** 9], dtype=torch.int32, device="cuda"), rows_per_count=4, max_rows=n)
    xq, xs, _ = matrix(1, n, C)
    wq, ws, _ = matrix(2, 2 * cout, C)
    x = rows(3, n, C, "bf16")
    y, z = (torch.full((n, C), 7.0, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    o = torch.full((n, cout), 7.0, dtype=torch.bfloat16, device="cuda")
    (aq, as_), (bq, bs), (gq, gs) = room(n, C), room(n, C), room(n, cout)
    api.sige_rows8_store(x, aq, as_, C, **kw)
    api.sige_rows8_load(xq, xs, y, C, **kw)
    api.sige_token_rms(x, C, y=z, q=bq, scales=bs, **kw)
    for form in range(8):
        with api.knobs(ROWS8_FORM=form):
            api.sige_rows8_linear(xq, xs, wq, ws, o, C, cout, **kw)
            if form < 4:
                api.sige_rows8_linear_gated(xq, xs, wq, ws, gq, gs, C, cout, **kw)
    torch.cuda.synchronize()
    for t in (y, z, o):
        assert (t == 7.0).all()
    for q, s, c in ((aq, as_, C), (bq, bs, C), (gq, gs, cout)):
        check_room(q, s, 0, c)


@pytest.mark.parametrize("kind", ["store", "rms", "linear"])
def test_offsets_beyond_32_bits(kind):
    """The last rows of tensors whose offsets do not fit 32 bits."""
    C, n = 8192, 2 ** 31 // 8192 + 300
    if kind == "linear":
        xq, xs, xv = matrix(1, 3, C)
        wq, ws, wv = matrix(2, 16, C, C ** -0.5)
        q, s = api.rows8(n, C)
        q[-3:], s[-3:] = xq, xs
        q[:-3], s[:-3] = 0, 0
        y = torch.empty(n, 16, dtype=torch.bfloat16, device="cuda")
        api.sige_rows8_linear(q, s, wq, ws, y, C, 16, n_rows=n)
        torch.cuda.synchronize()
        want, mag, cut = product(xv, wv, C)
        assert (np.abs(f64(y[-3:]) - want) <= C * 2.0 ** -24 * mag + cut + 2.0 ** -8 * (np.abs(want) + cut)).all() and (y[:-3] == 0).all()
        return
    x = torch.zeros(n, C, dtype=torch.bfloat16, device="cuda")
    x[-2:] = rows(1, 2, C, "bf16", 0)
    q, s = api.rows8(n, C)
    if kind == "store":
        api.sige_rows8_store(x, q, s, C, n_rows=n)
        y = torch.empty_like(x)
        api.sige_rows8_load(q, s, y, C, n_rows=n)
        torch.cuda.synchronize()
        same_codes(q[-2:], s[-2:], f64(x[-2:]), C)
        np.testing.assert_array_equal(f64(y[-2:]), ref.values(q[-2:].cpu().numpy(), s[-2:].cpu().numpy(), C))
    else:
        y = torch.empty_like(x)
        api.sige_token_rms(x, C, y=y, q=q, scales=s, n_rows=n)
        torch.cuda.synchronize()
        want = rms_expected(x[-2:], None, None, 1e-6, "bf16")[1]
        assert (np.abs(f64(y[-2:]) - want) <= (2.0 ** -8 + 2.0 ** -10) * np.abs(want)).all()
        close_codes(q[-2:], s[-2:], want, C * 2.0 ** -24 * np.abs(want), C)
    assert (y[:-2] == 0).all()


# ---- as they are used ----------------------------------------------------------------------------------

def feed_forward(x, indices, g, n_blocks, p, tiles, h, q, s, v, vs, y, full, C):
    """A feed-forward layer on the tokens of an edit, from the full tensor back into it."""
    api.sige_gather(x, g, indices, None, tiles, n_blocks=n_blocks)
    t, n = tiles.view(-1, C), n_blocks * g.block_h * g.block_w
    api.sige_token_rms(t, C, p["gamma"], 1e-6, q=q, scales=s, n_rows=n)
    api.sige_rows8_linear_gated(q, s, *p["first"], v, vs, C, 4 * C, bias=p["b1"], n_rows=n)
    api.sige_rows8_linear(v, vs, *p["second"], y, 4 * C, C, bias=p["b2"], base=t, n_rows=n)
    api.sige_scatter(y.view(tiles.shape), g, indices, None, full, n_blocks=n_blocks)


def layer(seed, C, dtype="bf16"):
    gen = torch.Generator().manual_seed(seed)
    r = lambda *shape: torch.randn(*shape, generator=gen, dtype=torch.float64)   # noqa: E731
    p = {"gamma": (1 + 0.1 * r(C)).float().cuda(), "b1": (0.1 * r(8 * C)).float().cuda(), "b2": (0.1 * r(C)).float().cuda()}
    for name, shape in (("first", (8 * C, C)), ("second", (C, 4 * C))):
        w = (r(*shape) / shape[1] ** 0.5).to(DT[dtype]).cuda()
        p[name] = api.rows8(*shape)
        api.sige_rows8_store(w, *p[name], shape[1], n_rows=shape[0])
    return p


def test_feed_forward_layer_of_an_edit():
    """Gather, norm, the gated product, the product with the residual, scatter: every stored tensor against its definition on what the call
    read; then captured into a graph and replayed on other edits, between eager calls."""
    C, side, nb = 72, 32, 6
    p = layer(0, C)
    g = api.geom(side, side, 4, 1, 1, 0)
    x = torch.randn(side, side, C, generator=torch.Generator().manual_seed(1)).bfloat16().cuda()
    pick = torch.tensor([3, 9, 20, 33, 40, 63])
    indices = torch.stack([pick // 8 * 4, pick % 8 * 4], 1).int().cuda()
    n = nb * 16
    tiles, y, full = torch.empty(nb, 4, 4, C).bfloat16().cuda(), torch.empty(n, C).bfloat16().cuda(), x.clone()
    q, s, v, vs = *api.rows8(n, C), *api.rows8(n, 4 * C)
    args = (x, indices, g, nb, p, tiles, None, q, s, v, vs, y, full, C)
    feed_forward(*args)
    torch.cuda.synchronize()
    t = f64(tiles.view(n, C))
    nrm = t / np.sqrt((t * t).mean(1, keepdims=True) + 1e-6) * f64(p["gamma"])
    close_codes(q, s, nrm, (C + 16) * 2.0 ** -24 * np.abs(nrm), C, "norm")
    val = lambda m, c: ref.values(m[0].cpu().numpy(), m[1].cpu().numpy(), c)   # noqa: E731
    want, mag, cut = product(val((q, s), C), val(p["first"], C), C)
    want, err = want + f64(p["b1"]), (C + 4) * 2.0 ** -24 * (mag + 1) + cut
    u, gt = want[:, :4 * C], want[:, 4 * C:]
    off = err[:, :4 * C] * (np.abs(ref.gate(gt, 0)) + 1.13 * err[:, 4 * C:]) + np.abs(u) * 1.13 * err[:, 4 * C:] + 2.0 ** -18 * np.abs(u * gt)
    close_codes(v, vs, u * ref.gate(gt, 0), off, 4 * C, "gated")
    want, mag, cut = product(val((v, vs), 4 * C), val(p["second"], 4 * C), 4 * C)
    want = want + f64(p["b2"]) + t
    bound = (4 * C + 4) * 2.0 ** -24 * (mag + np.abs(t) + 1) + cut
    assert (np.abs(f64(y) - want) <= bound + 2.0 ** -8 * (np.abs(want) + bound)).all()
    for i, (y0, x0) in enumerate(indices.tolist()):
        assert torch.equal(full[y0:y0 + 4, x0:x0 + 4], y.view(nb, 4, 4, C)[i])

    side_stream, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    side_stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=side_stream):
        feed_forward(*args)
    for k in range(4):
        x.copy_(torch.randn(side, side, C, generator=torch.Generator().manual_seed(10 + k)).bfloat16())
        indices.copy_(torch.tensor([[4 * ((i + k) % 8), 4 * ((3 * i + k) % 8)] for i in range(nb)]).int())
        full.copy_(x)
        graph.replay()
        torch.cuda.synchronize()
        got = full.clone()
        full.copy_(x)
        feed_forward(*args)
        torch.cuda.synchronize()
        assert torch.equal(got, full) and not torch.equal(full, x)


def test_two_streams_at_once():
    """The calls hold no state: the same layers on two streams at the same time, each with buffers of its own."""
    C, n = 320, 48
    p = layer(3, C)
    sets = []
    for k in range(2):
        x = rows(k, n, C, "bf16", 0)
        sets.append((x, *api.rows8(n, C), *api.rows8(n, 4 * C), torch.empty_like(x)))

    def run(x, q, s, v, vs, y):
        api.sige_token_rms(x, C, p["gamma"], q=q, scales=s, n_rows=n)
        api.sige_rows8_linear_gated(q, s, *p["first"], v, vs, C, 4 * C, gate=api.GATE_SILU, bias=p["b1"], n_rows=n)
        api.sige_rows8_linear(v, vs, *p["second"], y, 4 * C, C, base=x, n_rows=n)
    want = []
    for a in sets:
        run(*a)
        torch.cuda.synchronize()
        want.append(a[-1].clone())
        a[-1].zero_()
    streams = [torch.cuda.Stream() for _ in sets]
    torch.cuda.synchronize()
    for _ in range(20):
        for st, a in zip(streams, sets):
            with torch.cuda.stream(st):
                run(*a)
    torch.cuda.synchronize()
    for a, w in zip(sets, want):
        assert torch.equal(a[-1], w)


def test_recorded_calls():
    """Calls marshalled once and repeated."""
    C, n = 320, 5
    x = rows(0, n, C, "f16", 0)
    q, s = api.rows8(n, C)
    y = torch.empty_like(x)
    with api.record() as calls:
        api.sige_token_rms(x, C, q=q, scales=s, n_rows=n)
        api.sige_rows8_load(q, s, y, C, n_rows=n)
    torch.cuda.synchronize()
    want = y.clone()
    y.zero_()
    calls.run()
    torch.cuda.synchronize()
    assert len(calls) == 2 and torch.equal(y, want)


def test_one_row_of_as_many_channels_as_an_int_counts():
    """2^31 - 128 channels: chunks are counted without 2^31 - 128 + 511 becoming negative, and the row is what its blocks are as rows."""
    C = 2 ** 31 - 128
    n = C // 128
    x = torch.empty(1, C, dtype=torch.bfloat16, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(31)
    for i in range(0, C, 1 << 26):
        x[0, i:i + (1 << 26)].normal_(generator=g)
    q, s = api.rows8(1, C)
    api.sige_rows8_store(x, q, s, C, n_rows=1)
    bq, bs = api.rows8(n, 128)
    api.sige_rows8_store(x.view(n, 128), bq, bs, 128, n_rows=n)
    assert torch.equal(q.view(n, 128), bq) and torch.equal(s[0, :n], bs[:, 0]) and (s[0, n:] == 0).all()
    y = torch.empty_like(x)
    api.sige_rows8_load(q, s, y, C, n_rows=1)
    by = torch.empty(n, 128, dtype=torch.bfloat16, device="cuda")
    api.sige_rows8_load(bq, bs, by, 128, n_rows=n)
    assert torch.equal(y.view(n, 128), by)


def test_as_many_rows_as_a_launch_holds():
    """2^26 - 4 rows, the most that the calls take: the last of them in the store, the load and the norm."""
    C, n = 8, 2 ** 26 - 4
    x = torch.zeros(n, C, dtype=torch.bfloat16, device="cuda")
    x[-3:] = rows(26, 3, C, "bf16", 0)
    q, s = api.rows8(n, C)
    api.sige_rows8_store(x, q, s, C, n_rows=n)
    y = torch.empty_like(x)
    api.sige_rows8_load(q, s, y, C, n_rows=n)
    same_codes(q[-3:], s[-3:], f64(x[-3:]), C)
    np.testing.assert_array_equal(f64(y[-3:]), ref.values(q[-3:].cpu().numpy(), s[-3:].cpu().numpy(), C))
    assert (y[:-3] == 0).all()
    api.sige_token_rms(x, C, y=y, n_rows=n)
    want = rms_expected(x[-3:], None, None, 1e-6, "bf16")[1]
    assert (np.abs(f64(y[-3:]) - want) <= (2.0 ** -8 + 2.0 ** -10) * np.abs(want)).all() and (y[:-3] == 0).all()


@pytest.mark.parametrize("counted", [False, True])
def test_an_edit_without_blocks(counted):
    """Every call on tensors of no rows, also by a count on the device that such a program keeps."""
    C, cout = 320, 640
    kw = dict(n_rows=-1, count=torch.tensor([3], dtype=torch.int32, device="cuda"), rows_per_count=16) if counted else dict(n_rows=0)
    x, y, t = (torch.empty(0, C, dtype=torch.bfloat16, device="cuda") for _ in range(3))
    z = torch.empty(0, cout, dtype=torch.bfloat16, device="cuda")
    (q, s), (o, os_) = api.rows8(0, C), api.rows8(0, cout)
    w, ws = api.rows8(2 * cout, C)
    w.zero_(), ws.zero_()
    api.sige_rows8_store(x, q, s, C, **kw)
    api.sige_rows8_load(q, s, y, C, **kw)
    api.sige_token_rms(x, C, y=y, **kw)
    api.sige_token_rms(x, C, q=q, scales=s, **kw)
    api.sige_token_rms(x, C, residual=y, total=t, y=torch.empty(0, C + 8, dtype=torch.bfloat16, device="cuda"), q=q, scales=s, **kw)
    api.sige_rows8_linear(q, s, w, ws, z, C, cout, base=torch.empty(0, cout + 8, dtype=torch.bfloat16, device="cuda"), **kw)
    api.sige_rows8_linear_gated(q, s, w, ws, o, os_, C, cout, **kw)
    torch.cuda.synchronize()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n,C", [(8, 40), (8, 320), (9, 640), (8, 1288), (8, 4096), (8, 8192), (2060, 1032), (2060, 2048)])
def test_rms_rows_of_any_size(n, C, dtype):
    """Rows whose squares lie below or above what single precision holds, between others."""
    x = rows(C + n, n, C, dtype).clone()
    size = [0, -80, -120, -138 if dtype == "f32" else -130, 90, 118, -56, 0]
    for i, e in enumerate(size):
        x[i] = torch.ldexp(x[i].float(), torch.tensor(e, device="cuda")).to(DT[dtype])
    assert torch.isfinite(x).all()
    gamma = (torch.rand(C, generator=torch.Generator().manual_seed(C)) + 0.5).cuda()
    for gm, eps in ((None, 0.0), (gamma, 2.0 ** -160), (gamma, 2.0 ** -120), (None, 2.0 ** -81), (None, 2.0 ** -79), (gamma, 1e-6)):
        want = rms_expected(x, None, gm, float(np.float32(eps)), dtype)[1]
        rel = (C / 2 + 16) * 2.0 ** -24         # as in test_rms: powers of two add nothing
        y, (q, s) = torch.empty_like(x), room(n, C)
        api.sige_token_rms(x, C, gm, eps, y=y, q=q, scales=s, n_rows=n)
        torch.cuda.synchronize()
        # (where eps leaves values among single precision's smallest, both products round to its steps there, the first times gamma <= 1.5)
        tiny = 2.5 * 2.0 ** -150
        bound = (rel + torch.finfo(DT[dtype]).eps / 2 * (1 + rel)) * np.abs(want) + tiny + TINY[dtype]
        off = np.abs(f64(y) - want)
        assert (off <= bound).all(), (eps, np.argwhere(~(off <= bound))[:4].tolist())
        close_codes(q, s, want, rel * np.abs(want) + tiny, C, "norm")
        check_room(q, s, n, C)
    # in place behind a residual; the sum is the tensor that is normed
    z, res = x.clone(), torch.zeros_like(x)
    res[:, :8] = x[:, :8]
    h, want = rms_expected(x, res, None, 0.0, dtype)
    api.sige_token_rms(z, C, None, 0.0, residual=res, total=res, y=z, n_rows=n)
    torch.cuda.synchronize()
    np.testing.assert_array_equal(f64(res), h)
    assert (np.abs(f64(z) - want) <= (rel + torch.finfo(DT[dtype]).eps / 2 * (1 + rel)) * np.abs(want) + TINY[dtype]).all()


def test_rms_rows_of_any_size_that_are_not_finite():
    """A row of zeros without eps is 0 / 0; NaN and infinity beside numbers that overflow."""
    for C in (320, 640, 4096):
        x = torch.zeros(5, C, dtype=torch.float32, device="cuda")
        x[1], x[2], x[3], x[4] = 2.0 ** 120, 2.0 ** -100, 2.0 ** 100, 1.0
        x[1, 3], x[3, 5], x[2, 0] = float("inf"), float("nan"), 2.0 ** -101
        y = torch.empty_like(x)
        api.sige_token_rms(x, C, None, 0.0, y=y, n_rows=5)
        assert torch.isnan(y[0]).all() and torch.isnan(y[3]).all() and torch.isnan(y[1, 3])
        assert (torch.cat([y[1, :3], y[1, 4:]]) == 0).all()
        assert (y[4] == 1).all() and abs(y[2, 1].item() / y[2, 0].item() - 2) < 2.0 ** -22 and abs(y[2, 1].item() - 1) < 2.0 / C


@pytest.mark.parametrize("gate", [api.GATE_GELU, api.GATE_SILU])
@pytest.mark.parametrize("form", range(4))
def test_gates_far_below_zero(form, gate):
    """The activation relative to its own value, to the ends where that is nearly nothing: gates and values that come from the biases alone, every
    block of 128 channels with gates of one size, so that its scale is that of their values."""
    n, cin, cout = 3, 16, 128 * 192
    rng = np.random.default_rng(form + 8 * gate)
    lo, hi = (-12.9, 9.0) if gate == api.GATE_GELU else (-80.0, 40.0)
    g = (np.repeat(rng.uniform(lo, hi, cout // 128), 128) + rng.uniform(-0.05, 0.05, cout)).astype(np.float32)
    u = (rng.uniform(0.5, 2.0, cout) * rng.choice([-1.0, 1.0], cout)).astype(np.float32)
    x, xs, _ = matrix(3, n, cin)
    w, ws = torch.zeros(2 * cout, 128, dtype=torch.uint8, device="cuda"), torch.zeros(2 * cout, 4, dtype=torch.uint8, device="cuda")
    ws[:, 0] = 127
    q, s = room(n, cout)
    with api.knobs(ROWS8_FORM=form):
        api.sige_rows8_linear_gated(x, xs, w, ws, q, s, cin, cout, gate=gate, bias=torch.from_numpy(np.concatenate([u, g])).cuda(), n_rows=n)
    torch.cuda.synchronize()
    check_room(q, s, n, cout)
    d, z = g.astype(float), np.abs(g.astype(float))
    want = u * ref.gate(d, gate)
    # gelu: 1.7e-6 of the fit and its arithmetic (below 32 steps of 2^-24), and the exponent z * (z * c), |c| = 0.72, rounded twice: 2^-23 of itself, in powers of e
    # z^2 / 2 * 2^-23; silu: the exponent is rounded once, as its factor is: 2^-23 z; exp2 and reciprocal of the instruction set one step of 2^-23 each, four roundings
    rel = 2.0 ** -24 * (z * z + 40 if gate == api.GATE_GELU else 2 * z + 10)
    low, high = np.abs(want) * (1 - rel), np.abs(want) * (1 + rel)
    got, bytes_ = q.cpu().numpy()[:n, :cout], s.cpu().numpy()[:n, :cout // 128].astype(int)
    e = np.vectorize(ref.scale_exponent)
    assert (bytes_ - 127 >= e(low.reshape(-1, 128).max(1))).all() and (bytes_ - 127 <= e(high.reshape(-1, 128).max(1))).all()
    scale = 2.0 ** (np.repeat(bytes_, 128, 1) - 127.0)
    assert (got & 0x7f >= ref.nearest_code(low / scale)).all() and (got & 0x7f <= ref.nearest_code(high / scale)).all()
    assert ((got > 127) == (want < 0))[got & 0x7f != 0].all() and (got & 0x7f != 0).mean() > 0.95


def test_gated_product_with_weights_of_more_than_2_gib():
    """Gates that begin more than 2^31 bytes behind their values: every form, and more rows than the form for few of them takes."""
    cin, cout, wide = 640, 264, 2 ** 22 - 128
    x, xs, _ = matrix(41, 200, cin)
    w, ws, _ = matrix(42, 2 * cout, cin, cin ** -0.5)
    bias = torch.randn(2 * cout, generator=torch.Generator().manual_seed(43)).cuda()
    far = torch.empty(2 * cout, wide, dtype=torch.uint8, device="cuda")[:, :w.shape[1]]
    far.copy_(w)
    assert cout * wide + (cout - 1) * wide >= 2 ** 31
    for form in [-1] + list(range(4)):
        got = []
        for weights in (w, far):
            q, s = room(200, cout)
            with api.knobs(ROWS8_FORM=form):
                api.sige_rows8_linear_gated(x, xs, weights, ws, q, s, cin, cout, bias=bias, n_rows=200)
            check_room(q, s, 200, cout)
            got.append((q, s))
        assert torch.equal(got[0][0], got[1][0]) and torch.equal(got[0][1], got[1][1]), form
    # 2^20 rows: as the same rows 2^19 at a time by weights without gaps
    n, cin = 2 ** 20, 128
    g = torch.Generator(device="cuda").manual_seed(44)
    t = torch.randn(n, cin, generator=g, device="cuda", dtype=torch.float32).bfloat16()
    x, xs = api.rows8(n, cin)
    api.sige_rows8_store(t, x, xs, cin, n_rows=n)
    near = far[:, :cin].contiguous()
    q, s = api.rows8(n, cout)
    api.sige_rows8_linear_gated(x, xs, far, ws, q, s, cin, cout, bias=bias, n_rows=n)
    for i in (0, n // 2):
        q2, s2 = api.rows8(n // 2, cout)
        api.sige_rows8_linear_gated(x[i:i + n // 2], xs[i:i + n // 2], near, ws, q2, s2, cin, cout, bias=bias, n_rows=n // 2)
        assert torch.equal(q[i:i + n // 2], q2) and torch.equal(s[i:i + n // 2], s2)


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
def test_more_tiles_of_128_than_compute_units(dtype):
    """The form with four blocks on their way, on more tiles than compute units with more blocks than that: the bits of the form with two."""
    for n, cin, cout in ((2100, 520, 2200), (2176, 1160, 2304)):
        x, w = drawn(n, n, cin), drawn(cout, cout, cin, cin ** -0.5)
        bias, base = torch.randn(cout, device="cuda"), torch.randn(n, cout, device="cuda").to(DT[dtype])
        y = []
        for form in (5, 6):
            y.append(torch.full((n + 1, cout + 8), 7.0, dtype=DT[dtype], device="cuda"))
            with api.knobs(ROWS8_FORM=form):
                api.sige_rows8_linear(*x, *w, y[-1][:n, :cout], cin, cout, bias=bias, base=base, n_rows=n)
        assert torch.equal(y[0], y[1]) and (y[1][n] == 7.0).all() and (y[1][:, cout:] == 7.0).all()
        xv, wv = on_gpu(*x, cin), on_gpu(*w, cin)
        want = xv @ wv.t() + bias.double() + base.double()
        bound = (cin + 4) * 2.0 ** -24 * (xv.abs() @ wv.abs().t() + bias.double().abs() + base.double().abs()) + (0 if dtype == "f32" else cut_of(xv, wv))
        bound = bound + torch.finfo(DT[dtype]).eps / 2 * (want.abs() + bound) + TINY[dtype]
        assert ((y[1][:n, :cout].double() - want).abs() <= bound).all()

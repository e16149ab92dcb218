"""The attention on the cache in 4 bits at the ends of its numbers, against float64 (tests/cache4_oracle.py)."""
import numpy as np
import pytest
import torch

import cache4_oracle as ref
from paper_2211_02048_amd import api
from test_gpu_cache4 import DT, attend, case, close, f64, forms, some_ranges

pytestmark = pytest.mark.gpu


def cache_of(k, v, dtype, capacity):
    """A cache of the rows k, v [T, heads, d] (float64, numbers that it holds exactly), and what it holds."""
    T, heads, d = k.shape
    cache = np.random.default_rng(T).integers(0, 256, api.sige_cache4_bytes(heads, d, capacity), dtype=np.uint8)
    for which, x in enumerate((k, v)):
        code, byte = ref.quantise(x, DT[dtype])
        for t in range(T):
            ref.put(cache, heads, d, capacity, t, code[t], byte[t], which)
    return cache, ref.read(cache, heads, d, capacity, T, 0), ref.read(cache, heads, d, capacity, T, 1)


def near(o, want, mag, dtype, T, what, logits=0.0):
    """As test_gpu_cache4.close for logits whose error is known (none: they are exact): |o - want| <= (p + s) sum_t p_t |v_t| + r |want| with p the rounding
    of the probabilities in numerator and denominator (single precision: three parts), s the exponential's 2^-21 in both and the
    T terms of both sums, twice the logits' error, r the rounding of the result."""
    eps = torch.finfo(DT[dtype]).eps
    p = eps if dtype != "f32" else 2.0 ** -22
    bound = (p + 2.0 ** -20 + T * 2.0 ** -23 + 2 * logits) * mag + eps / 2 * np.abs(want) + (2.0 ** -25 if dtype == "f16" else 1e-30)
    got = f64(o).reshape(want.shape)
    assert np.isfinite(got).all(), f"{what}: {int((~np.isfinite(got)).sum())} of {got.size} are no numbers"
    assert (np.abs(got - want) <= bound).all(), f"{what}: worst {np.max(np.abs(got - want) / bound):.2f} of the bound"


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("d", [24, 40, 64, 96, 128, 200, 256])
def test_logits_of_any_size(d, dtype):
    """Logits up to the end of single precision beside ordinary ones.  Keys and queries have one channel, so that every logit is
    exact; tokens of the same key share a row's probability equally, those of another one lie far below in the rows of large logits.
    The rows of ordinary logits give bit for bit what they give beside rows of zeros."""
    heads, nq, T, scale = 2, 40, 300, 0.125
    rng = np.random.default_rng(d)
    grid = np.array([-6.0, -4.0, -1.5, 0.0, 0.5, 3.0, 6.0])
    e = 13 if dtype == "f16" else 0
    k = np.zeros((T, heads, d))
    k[..., d // 2] = np.sort(rng.choice(grid, (T, heads)), axis=0) * 2.0 ** e          # (the maximum moves from chunk to chunk)
    v = rng.standard_normal((T, heads, d))
    # queries of 8 bits; largest logits about 1 and 10^6 .. 10^8 (fp16), 10^6 .. 10^37
    sizes = [1.0, 1e6, 5e6, 8e6, 1.3e7, 3e7, 1e8, 3e8] if dtype == "f16" else [1.0, 1e7, 1e8, 2e9, 1e10, 1e15, 1e25, 1e37]
    size = np.array(sizes)[np.arange(nq) % 8] / (6 * 2.0 ** e * scale)
    q = np.zeros((nq, heads, d))
    q[..., d // 2] = (size * rng.choice([-1.0, 1.0], nq))[:, None] * (1 + rng.integers(0, 64, (nq, heads)) / 128)
    q[..., d // 2] *= np.where(np.abs(q[..., d // 2]) > (60000 if dtype == "f16" else 1e38), 0.5, 1.0)
    qt = torch.from_numpy(q.reshape(nq, heads * d)).to(DT[dtype]).cuda()
    q = f64(qt).reshape(nq, heads, d)
    cap = T + 9
    cache, k, v = cache_of(k, v, dtype, cap)
    cache = torch.from_numpy(cache).cuda()
    ordinary = torch.from_numpy(np.arange(nq) % 8 == 0).cuda()
    alone = torch.where(ordinary[:, None], qt, torch.zeros_like(qt))
    for ranges in (None, some_ranges(nq, T, d)):
        want, mag = ref.attention(q, k, v, scale, ranges)
        for many in forms(dtype):
            for ws, wgs in ((True, None), (False, None), (True, 40)):
                with api.knobs(CACHE4_MANY=many, ATTN_WGS=wgs):
                    o = attend(qt, cache, cap, T, heads, d, scale, ranges, ws)
                    near(o, want, mag, dtype, T, f"form {many}, workspace {ws}, {wgs} workgroups")
                    assert torch.equal(o[ordinary], attend(alone, cache, cap, T, heads, d, scale, ranges, ws)[ordinary])


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("d", [40, 64, 128])
def test_large_logits_of_all_channels(d, dtype):
    """Queries and keys of one direction and of any, logits of 10^7, 10^8 and (beyond fp16) 10^10: which of two tokens that are
    closer than the logits' rounding counts more is open, but every value is a mean of the values that the row sees."""
    heads, nq, T, cap = 2, 70, 500, 500
    scale = d ** -0.5
    rng = np.random.default_rng(d)
    for size in (1e7, 1e8) if dtype == "f16" else (1e7, 1e8, 1e10):
        k, v = rng.standard_normal((T, heads, d)), rng.standard_normal((T, heads, d))
        k[: T // 2] = np.sign(k[0]) * (1 + 0.3 * rng.random((T // 2, heads, d)))
        each = (size / (scale * d)) ** 0.5                     # a channel of a query and of a key
        k *= each
        q = np.where(np.arange(nq)[:, None, None] % 2 == 0, np.sign(k[:1]) * (1 + rng.random((nq, heads, d))), rng.standard_normal((nq, heads, d))) * each
        to = lambda x: torch.from_numpy(x.reshape(len(x), -1)).to(DT[dtype]).cuda()    # noqa: E731
        qt, kt, vt = to(q), to(k), to(v)
        assert torch.isfinite(qt).all() and torch.isfinite(kt).all()
        cache = torch.zeros(api.sige_cache4_bytes(heads, d, cap), dtype=torch.uint8, device="cuda")
        api.sige_cache4_store(kt, vt, cache, cap, heads, d, n_rows=T)
        torch.cuda.synchronize()
        held = ref.read(cache.cpu().numpy(), heads, d, cap, T, 1)
        lo, hi = held.min(0), held.max(0)
        room = 2 * torch.finfo(DT[dtype]).eps * np.maximum(np.abs(lo), np.abs(hi))
        for many in forms(dtype):
            for ws in (True, False):
                with api.knobs(CACHE4_MANY=many):
                    o = f64(attend(qt, cache, cap, T, heads, d, scale, None, ws)).reshape(nq, heads, d)
                assert np.isfinite(o).all(), f"{size}, form {many}: {int((~np.isfinite(o)).sum())} of {o.size} are no numbers"
                assert (o >= lo - room).all() and (o <= hi + room).all()


@pytest.mark.parametrize("d", [24, 64, 96, 256])
def test_queries_at_the_end_of_single_precision(d):
    """Queries up to the largest float, beyond the largest number of bf16, on keys so small that the logits are ordinary."""
    heads, nq, T = 2, 33, 50
    rng = np.random.default_rng(d)
    most = float(torch.finfo(torch.float32).max)
    k = np.zeros((T, heads, d))
    at = [0, d // 2, d - 1]
    k[..., at] = rng.choice([-6.0, -2.0, -0.5, 0.5, 1.0, 4.0], (T, heads, 3)) * 2.0 ** -125
    v = rng.standard_normal((T, heads, d))
    q = np.zeros((nq, heads, d))
    q[..., at] = rng.choice([most, -most, 3.4e38, 3.397e38, 3.39e38, 1e38, -3.0], (nq, heads, 3))
    qt = torch.from_numpy(q.reshape(nq, heads * d)).float().cuda()
    q = f64(qt).reshape(nq, heads, d)
    cache, k, v = cache_of(k, v, "f32", T)
    want, mag = ref.attention(q, k, v, 0.125)
    o = attend(qt, torch.from_numpy(cache).cuda(), T, T, heads, d, 0.125)
    # (nine products - three channels, three parts - are added in fp32: 2^-24 of at most 3 * 6 2^-125 * 2^128 / 8 = 18 each time)
    near(o, want, mag, "f32", T, "the largest queries", logits=9 * 18 * 2.0 ** -24)
    qt[5, 1] = float("inf")
    qt[6, d] = float("nan")
    o = attend(qt, torch.from_numpy(cache).cuda(), T, T, heads, d, 0.125).view(nq, heads, d)
    assert torch.isnan(o[5, 0]).all() and torch.isnan(o[6, 1]).all()
    assert torch.isfinite(o[:5]).all() and torch.isfinite(o[7:]).all()


def in_parts(x, n):
    """What n bf16 numbers hold of x, each the rounding of what the ones before left."""
    left, held = torch.from_numpy(x).clone(), torch.zeros(x.shape, dtype=torch.float64)
    for _ in range(n):
        part = left.bfloat16().double()
        held, left = held + part, left - part
    return held.numpy()


@pytest.mark.parametrize("d", [8, 24, 40, 64, 96, 128, 160, 200, 248, 256])
def test_single_precision_keeps_24_bits(d):
    """Queries that differ in their last 8 bits alone, keys of 2^18 in one channel each: exact logits of unlike tokens less than 3
    apart, which the first 16 bits do not tell; values of both signs, so that what a probability loses is left over.  The bound
    refuses two parts of a query, and two of a probability."""
    heads, nq, T = 2, 70, 5
    rng = np.random.default_rng(d)
    k = np.zeros((T, heads, d))
    at = np.arange(T) * d // T
    k[np.arange(T), :, at] = 2.0 ** 18
    v = rng.choice([-1.0, 1.0], (T, heads, d))
    q = rng.standard_normal((nq, heads, d))
    q[..., at] = 1 + rng.integers(0, 2 ** 15, (nq, heads, 1)) * 2.0 ** -15 + rng.integers(0, 96, (nq, heads, T)) * 2.0 ** -23
    qt = torch.from_numpy(q.reshape(nq, heads * d)).float().cuda()
    q = f64(qt).reshape(nq, heads, d)
    cache, k, v = cache_of(k, v, "f32", T)
    want, mag = ref.attention(q, k, v, 1.0)
    near(attend(qt, torch.from_numpy(cache).cuda(), T, T, heads, d, 1.0), want, mag, "f32", T, "24 bits")
    with pytest.raises(AssertionError, match="of the bound"):
        near(torch.from_numpy(ref.attention(in_parts(q, 2), k, v, 1.0)[0]), want, mag, "f32", T, "two parts of a query")
    s = np.einsum("ihc,thc->iht", q, k)
    p = np.exp(s - s.max(-1, keepdims=True))
    fewer = np.einsum("iht,thc->ihc", in_parts(p, 2), v) / p.sum(-1)[..., None]
    with pytest.raises(AssertionError, match="of the bound"):
        near(torch.from_numpy(fewer), want, mag, "f32", T, "two parts of a probability")


@pytest.mark.parametrize("dtype,nq,T,heads,d,many", [("bf16", 2100, 700, 8, 64, 1), ("f16", 1500, 1100, 12, 40, 1), ("bf16", 4200, 16400, 2, 96, 1), ("f16", 4100, 20000, 1, 128, 1),
                                                     ("bf16", 2050, 12000, 2, 160, 1), ("f16", 1300, 700, 5, 64, 0), ("bf16", 4200, 8200, 2, 96, 0), ("f16", 1000, 16400, 1, 128, 0),
                                                     ("bf16", 600, 9000, 1, 160, 0)])
def test_which_form_a_call_takes(dtype, nq, T, heads, d, many):
    """Half types take the form for many queries where heads of up to 64 have more tiles of 32 queries than compute units (256), and where
    tiles x tokens x d^2 of larger ones passes 2^35: bit for bit what the knob makes of the call, and not what it makes the other way
    (up to 64: the forms differ in a workgroup's waves, up to 256 and from 513 tiles on); every row against float64 on the GPU."""
    tiles = -(-nq // 32) * heads
    assert (tiles > 256 if d <= 64 else tiles * T * d * d >= 2 ** 35) == bool(many)
    q, cache, cap, k, v = case(7, nq, T, heads, d, dtype)
    k, v = torch.from_numpy(k).cuda(), torch.from_numpy(v).cuda()
    scale = d ** -0.5
    o = attend(q, cache, cap, T, heads, d, scale)
    forced = {}
    for m in (0, 1):
        with api.knobs(CACHE4_MANY=m):
            forced[m] = attend(q, cache, cap, T, heads, d, scale)
    assert torch.equal(o, forced[many]) and not torch.equal(o, forced[1 - many])
    q64 = q.double().view(nq, heads, d)
    for h in range(heads):
        p = torch.softmax(q64[:, h] @ k[:, h].t() * scale, -1)
        want, mag = (p @ v[:, h]).cpu().numpy()[:, None], ((p + 2.0 ** -30) @ v[:, h].abs()).cpu().numpy()[:, None]
        close(o[:, h * d:(h + 1) * d], want, mag, q64[:, h:h + 1].cpu().numpy(), k[:, h:h + 1].cpu().numpy(), scale, dtype, T, f"{nq} of {T} x {d}")

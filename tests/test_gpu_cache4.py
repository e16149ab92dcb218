"""The cache of keys and values in 4 bits on the GPU: store, load and the attention that reads it, against their definitions in
float64 (tests/cache4_oracle.py)."""
import math

import numpy as np
import pytest
import torch

import cache4_oracle as ref
from paper_2211_02048_amd import api

pytestmark = pytest.mark.gpu
DT = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
HEADS_OF = [8, 16, 24, 40, 64, 72, 80, 96, 128, 160, 200, 216, 248, 256]


def f64(t):
    return t.detach().cpu().double().numpy()


def rows(seed, n, heads, d, dtype, ld=None):
    """[n, heads * d] rows of a wider tensor, values over several magnitudes, N(0, 1) times a size per channel."""
    rng = np.random.default_rng(seed)
    x = rng.standard_normal((n, heads * d)) * np.exp(rng.standard_normal(heads * d))
    t = torch.zeros((n, ld or heads * d), dtype=DT[dtype])
    t[:, :heads * d] = torch.from_numpy(x)
    return t.cuda()[:, :heads * d]


def garbage(nbytes, seed=5):
    """A cache nobody initialised: any bytes, those that stand for no number among them."""
    return torch.from_numpy(np.random.default_rng(seed).integers(0, 256, nbytes, dtype=np.uint8)).cuda()


def same_values(got, want, heads, d, capacity):
    """Two caches hold the same values and scale bytes (a code of -0 is 0)."""
    for a, b in zip(ref.views(got, heads, d, capacity), ref.views(want, heads, d, capacity)):
        for x, y in zip(a, b):
            for u, v in zip(x[:2], y[:2]):
                if u is not None:
                    lo = lambda c: np.where((c & 15) == 8, c & 0xF0, c)                # noqa: E731
                    hi = lambda c: np.where((c >> 4) == 8, c & 0x0F, c)                # noqa: E731
                    assert np.array_equal(hi(lo(u)), hi(lo(v)))
            assert np.array_equal(x[2], y[2])


def expected(before, k, v, heads, d, capacity, tokens, dtype):
    """The cache's bytes after rows k, v went to `tokens` (-1: nowhere)."""
    want = before.cpu().numpy().copy()
    for which, x in enumerate((k, v)):
        code, byte = ref.quantise(f64(x).reshape(-1, heads, d), DT[dtype])
        for r, t in enumerate(tokens):
            if 0 <= t < capacity:
                ref.put(want, heads, d, capacity, t, code[r], byte[r], which)
    return want


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("d", HEADS_OF)
def test_store_and_load(d, dtype):
    """Rows in any slots, some of them nowhere; every byte of the other tokens stays; what is read back is what was stored."""
    heads, n, capacity = 3, 37, 61
    k, v = rows(d, n, heads, d, dtype, ld=heads * d + 16), rows(d + 1, n, heads, d, dtype)
    slots = np.random.default_rng(d).permutation(capacity)[:n].astype(np.int32)
    slots[[3, 20]] = -1, capacity
    cache = garbage(api.sige_cache4_bytes(heads, d, capacity))
    want = expected(cache, k, v, heads, d, capacity, slots, dtype)
    api.sige_cache4_store(k, v, cache, capacity, heads, d, slots=torch.from_numpy(slots).cuda(), n_rows=n)
    torch.cuda.synchronize()
    same_values(cache.cpu().numpy(), want, heads, d, capacity)
    there = np.array([s for s in slots if 0 <= s < capacity])
    for which, x in enumerate((k, v)):
        out = torch.full((capacity + 1, heads * d + 8), 7.0, dtype=DT[dtype], device="cuda")
        kw = dict(k=out[:capacity, :heads * d], v=None) if which == 0 else dict(k=None, v=out[:capacity, :heads * d])
        api.sige_cache4_load(cache, capacity, heads, d, **kw)
        torch.cuda.synchronize()
        all_ = ref.read(want, heads, d, capacity, capacity, which, 140 if dtype == "f16" else 252)
        assert np.array_equal(f64(out)[there, :heads * d].reshape(-1, heads, d), all_[there])
        assert (out[capacity] == 7.0).all() and (out[:, heads * d:] == 7.0).all()


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
def test_store_rounds_to_the_nearest(dtype):
    """Values on and beside the borders between neighbours, at several scales; the type's largest and smallest numbers, zeros,
    infinities and NaN."""
    td = DT[dtype]
    heads, d = 1, 32
    eps = torch.finfo(td).eps
    tests = []
    for e in (-3, 0, 5):
        for top in (6.0, 3.5, 4.0, 5.0, 3.0 * (1 + eps)):
            v = [0.0, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0]
            v += [x * (1 + eps) for x in v[1:]] + [x * (1 - eps) for x in v[1:]]
            v = [min(x, top) for x in v] + [top] + [-x for x in (0.25, 0.75, 1.25, 2.5)] + [-min(5.0, top), -0.0, 0.3, -0.1]
            tests.append(([x * 2.0 ** e for x in v] + [0.0])[:32])
    big, tiny = torch.finfo(td).max, torch.finfo(td).tiny
    tests += [[big, -big, big / 2, big / 7, big / 20] + [0.0] * 27, [0.0] * 32, [-0.0] * 32, [tiny, -tiny, tiny / 2, 3 * tiny] + [0.0] * 28,
              [tiny * 40] * 32, [float("inf")] + [1.0] * 31, [1.0] * 31 + [float("nan")], [-float("inf")] * 32]
    k = torch.tensor(tests, dtype=torch.float64).to(td).cuda()
    n = len(tests)
    cache = garbage(api.sige_cache4_bytes(heads, d, n))
    want = expected(cache, k, k, heads, d, n, range(n), dtype)
    api.sige_cache4_store(k, k, cache, n, heads, d, n_rows=n)
    out = torch.empty_like(k)
    api.sige_cache4_load(cache, n, heads, d, out, None)
    torch.cuda.synchronize()
    same_values(cache.cpu().numpy(), want, heads, d, n)
    np.testing.assert_array_equal(f64(out), ref.read(want, heads, d, n, n, 0)[:, 0])
    assert torch.isfinite(out[:-3]).all() and torch.isnan(out[-3:]).all()


@pytest.mark.parametrize("dtype,d,b,H,W,first", [("bf16", 40, 4, 18, 10, 0), ("f16", 80, 8, 20, 20, 7), ("f32", 72, 3, 9, 9, 100)])
def test_store_blocks(dtype, d, b, H, W, first):
    """Stacked tokens of listed blocks, some of which stick out of the map; the count on the host and on the device; rows past the
    count and tokens of other blocks stay."""
    heads, capacity = 2, first + H * W + 3
    g = api.geom(H, W, b, 1, 1, 0)
    gy, gx = -(-H // b), -(-W // b)
    pick = np.unique(np.r_[np.random.default_rng(d).permutation(gy * gx)[:5], gy * gx - 1])
    blocks = np.stack([pick // gx * b, pick % gx * b], 1).astype(np.int32)
    n = len(blocks)
    idx = torch.full((n + 2, 2), 0, dtype=torch.int32)
    idx[:n] = torch.from_numpy(blocks)
    k, v = (rows(s, (n + 2) * b * b, heads, d, dtype) for s in (1, 2))
    tokens = []
    for y0, x0 in blocks:
        for p in range(b * b):
            y, x = y0 + p // b, x0 + p % b
            tokens.append(first + y * W + x if y < H and x < W else -1)
    before = garbage(api.sige_cache4_bytes(heads, d, capacity))
    want = expected(before, k[:n * b * b], v[:n * b * b], heads, d, capacity, tokens, dtype)
    for n_blocks in (n, -1):
        cache = before.clone()
        api.sige_cache4_store_blocks(k, v, cache, capacity, heads, d, g, idx.cuda(), torch.tensor([n], dtype=torch.int32, device="cuda"),
                                     n_blocks=n_blocks, first=first)
        torch.cuda.synchronize()
        same_values(cache.cpu().numpy(), want, heads, d, capacity)


def test_store_by_device_count():
    heads, d, n, capacity = 2, 64, 50, 30
    k, v = rows(1, n, heads, d, "f16"), rows(2, n, heads, d, "f16")
    for count, per in ((3, 8), (7, 8), (0, 8)):
        cache = garbage(api.sige_cache4_bytes(heads, d, capacity))
        # 24 rows; 50 rows (of 56), of which those past the capacity are not stored; none
        want = expected(cache, k, v, heads, d, capacity, [6 + r if r < min(count * per, n) else -1 for r in range(n)], "f16")
        api.sige_cache4_store(k, v, cache, capacity, heads, d, first=6, count=torch.tensor([count], dtype=torch.int32, device="cuda"),
                              rows_per_count=per)
        torch.cuda.synchronize()
        same_values(cache.cpu().numpy(), want, heads, d, capacity)


# ---- attention -----------------------------------------------------------------------------------------

def close(o, want, mag, q, k, scale, dtype, T, what):
    """|o - want| <= (p + s) sum_t p_t |v_t| + r |want| with, all derived from the arithmetic:
    p  the rounding of the probabilities to the compute type, eps / 2 each in the numerator and as much in the denominator that adds
       them (single precision: three parts, 2^-24),
    s  the logits' error and the sums': d products and T terms added in fp32, (d + 4) 2^-24 scale sum |q k|, at most
       scale max|q| max|k| d, twice (numerator and denominator), the exponential's 2^-21, and T 2^-24,
    r  the rounding of the result, eps / 2;
    fp16 has no more bits below 2^-14: a result there is off by 2^-25, a probability (the largest counts 2^15) by 2^-40, which the
    2^-30 beside every p_t times p = 2^-10 stand for."""
    td = DT[dtype]
    eps = torch.finfo(td).eps
    p = eps if dtype != "f32" else 2.0 ** -22
    with np.errstate(invalid="ignore"):
        top = scale * np.nanmax(np.abs(q)[:, :, None, :] @ np.nanmax(np.abs(k), 0)[None, :, :, None]) if T else 0.0
    s = 2 * (q.shape[-1] + 4) * 2.0 ** -24 * top + 2.0 ** -20 + T * 2.0 ** -23
    bound = (p + s) * mag + eps / 2 * np.abs(want) + (2.0 ** -25 if dtype == "f16" else 1e-30)
    got = f64(o).reshape(want.shape)
    assert np.array_equal(np.isnan(got), np.isnan(want)), f"{what}: other places are NaN"
    ok = np.isnan(want) | (np.abs(got - want) <= bound)
    assert ok.all(), f"{what}: {int((~ok).sum())} of {ok.size} off, worst {np.nanmax(np.abs(got - want) / bound):.2f} of the bound"


def case(seed, nq, T, heads, d, dtype, capacity=None):
    capacity = T + 5 if capacity is None else capacity
    q = rows(seed, nq, heads, d, dtype)
    cache = garbage(api.sige_cache4_bytes(heads, d, capacity), seed)
    if T:
        k, v = rows(seed + 1, T, heads, d, dtype), rows(seed + 2, T, heads, d, dtype)
        api.sige_cache4_store(k, v, cache, capacity, heads, d, n_rows=T)
    torch.cuda.synchronize()
    c = cache.cpu().numpy()
    return q, cache, capacity, ref.read(c, heads, d, capacity, T, 0), ref.read(c, heads, d, capacity, T, 1)


def attend(q, cache, capacity, T, heads, d, scale, ranges=None, ws=True):
    nq = q.shape[0]
    o = torch.full((nq + 1, heads * d + 16), 7.0, dtype=q.dtype, device="cuda")
    nb = api.sige_cache4_attn_workspace_bytes(nq, T, heads, d)
    w = torch.full((nb // 4,), float("nan"), dtype=torch.float32, device="cuda") if ws and nb else None
    r = None if ranges is None else torch.from_numpy(np.ascontiguousarray(ranges, dtype=np.int32)).cuda()
    api.sige_cache4_attn(q, cache, capacity, o[:nq, :heads * d], scale, T=T, heads=heads, d=d, ranges=r, workspace=w)
    torch.cuda.synchronize()
    assert (o[nq] == 7.0).all() and (o[:, heads * d:] == 7.0).all(), "written outside the rows"
    return o[:nq, :heads * d]


SIZES = [(1, 1), (1, 700), (5, 33), (16, 320), (33, 64), (70, 65), (130, 257)]


def forms(dtype):
    """The forms of a call: by its own rule, that for few queries, that for many (half types)."""
    return (None,) if dtype == "f32" else (None, 0, 1)


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("d", HEADS_OF)
def test_attention(d, dtype):
    heads = 2
    for nq, T in SIZES:
        q, cache, cap, k, v = case(d + nq, nq, T, heads, d, dtype)
        scale = 1 / math.sqrt(d)
        want, mag = ref.attention(f64(q).reshape(nq, heads, d), k, v, scale)
        for many in forms(dtype):
            for ws in (True, False):
                with api.knobs(CACHE4_MANY=many):
                    o = attend(q, cache, cap, T, heads, d, scale, ws=ws)
                close(o, want, mag, f64(q).reshape(nq, heads, d), k, scale, dtype, T, f"{nq} of {T} x {d}, form {many}, workspace {ws}")


def some_ranges(nq, T, seed):
    """Requests of unlike lengths, rows that see one token, the first, the last, all, nothing, or what is not there."""
    rng = np.random.default_rng(seed)
    r = np.sort(rng.integers(0, T + 1, (nq, 2)), axis=1)
    special = [(0, 0), (T, T), (5, 3), (0, 1), (T - 1, T), (0, T), (-9, T + 9), (T + 3, T + 8), (-5, 0), (T // 2, T // 2 + 1)]
    for i, s in enumerate(special):
        if i < nq:
            r[(i * 7) % nq] = s
    return r


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("nq,T,heads,d", [(10, 50, 2, 64), (40, 1000, 2, 40), (150, 300, 1, 128), (300, 2100, 2, 72), (65, 129, 3, 256), (64, 31, 1, 8)])
def test_attention_ranges(nq, T, heads, d, dtype):
    q, cache, cap, k, v = case(nq, nq, T, heads, d, dtype)
    ranges = some_ranges(nq, T, d)
    scale = 1 / math.sqrt(d)
    q64 = f64(q).reshape(nq, heads, d)
    want, mag = ref.attention(q64, k, v, scale, ranges)
    # every row sees the tokens up to its own (a row per token of the last ones)
    own = np.stack([np.zeros(nq), np.minimum(np.arange(nq) + max(T - nq, 0) + 1, T)], 1).astype(int)
    want_own, mag_own = ref.attention(q64, k, v, scale, own)
    for many in forms(dtype):
        with api.knobs(CACHE4_MANY=many):
            for ws in (True, False):
                o = attend(q, cache, cap, T, heads, d, scale, ranges, ws)
                close(o, want, mag, q64, k, scale, dtype, T, f"ranges, form {many}, workspace {ws}")
                empty = np.array([max(b, 0) >= min(e, T) for b, e in ranges])
                assert empty.any() and (o[torch.from_numpy(empty).cuda()] == 0).all()
            # no row sees anything
            o = attend(q, cache, cap, T, heads, d, scale, np.zeros((nq, 2)))
            assert (o == 0).all()
            close(attend(q, cache, cap, T, heads, d, scale, own), want_own, mag_own, q64, k, scale, dtype, T, "up to its own token")


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("nq,heads,T,d", [(1030, 8, 3, 128), (1030, 8, 77, 40), (1030, 9, 200, 80), (830, 20, 77, 64), (830, 20, 200, 24), (820, 21, 77, 160),
                                          (860, 40, 70, 40), (860, 40, 77, 96), (350, 97, 90, 72), (400, 24, 130, 256)])
def test_attention_of_many_rows_and_few_tokens(nq, heads, T, d, dtype):
    """More workgroups than compute units: fewer waves in each, down to one."""
    q, cache, cap, k, v = case(nq, nq, T, heads, d, dtype)
    scale = 1 / math.sqrt(d)
    q64 = f64(q).reshape(nq, heads, d)
    want, mag = ref.attention(q64, k, v, scale)
    close(attend(q, cache, cap, T, heads, d, scale), want, mag, q64, k, scale, dtype, T, "all tokens")
    ranges = some_ranges(nq, T, d)
    want, mag = ref.attention(q64, k, v, scale, ranges)
    close(attend(q, cache, cap, T, heads, d, scale, ranges), want, mag, q64, k, scale, dtype, T, "ranges")


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("nq,heads,T,d,wgs", [(70, 1, 3000, 40, None), (70, 1, 3000, 40, 40), (300, 2, 2500, 64, 300), (140, 2, 2100, 160, 64), (40, 1, 1000, 248, 9)])
def test_attention_of_ranges_far_apart(nq, heads, T, d, wgs, dtype):
    """Neighbouring rows see parts of the cache with long stretches between them that nobody sees; the splits share out what a tile of
    rows spans."""
    q, cache, cap, k, v = case(d, nq, T, heads, d, dtype)
    i = np.arange(nq)
    ranges = np.stack([i % 3 * 900 + i % 7, np.minimum(i % 3 * 900 + 30 + i % 50, T)], 1)
    ranges[32:64] = (T - 5, T)                    # (a tile of its own: the last chunk alone)
    ranges[3] = (0, 0)
    scale = 1 / math.sqrt(d)
    q64 = f64(q).reshape(nq, heads, d)
    want, mag = ref.attention(q64, k, v, scale, ranges)
    for many in forms(dtype):
        for ws in (True, False):
            with api.knobs(CACHE4_MANY=many, ATTN_WGS=wgs):
                o = attend(q, cache, cap, T, heads, d, scale, ranges, ws)
            close(o, want, mag, q64, k, scale, dtype, T, f"far apart, form {many}, workspace {ws}")


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("nq,d", [(3, 64), (20, 40), (100, 64), (100, 40), (90, 160)])
def test_attention_of_tokens_that_are_no_numbers(nq, d, dtype):
    """Tokens whose keys, or whose values in one group, are not finite: NaN for the rows that see them (values: in that group's
    channels), nothing for the others, which see their part of the same chunk."""
    heads, T, cap = 2, 200, 200
    q, cache, cap, k, v = case(d, nq, T, heads, d, dtype, cap)
    c = cache.cpu().numpy().copy()
    views = ref.views(c, heads, d, cap)
    views[0][0][2][70, 0] = 255                # a key of the first head
    views[1][1][2][75, (d - 1) // 32] = 255    # the last group of a value of the second
    views[1][1][2][130, 0] = 253
    cache = torch.from_numpy(c).cuda()
    k, v = ref.read(c, heads, d, cap, T, 0), ref.read(c, heads, d, cap, T, 1)
    scale = 1 / math.sqrt(d)
    ranges = np.stack([np.arange(nq) % 9 * 10, 72 + np.arange(nq) * 7 % 129], 1)
    ranges[::5] = (76, 130)
    q64 = f64(q).reshape(nq, heads, d)
    for r in (ranges, None, np.tile([0, 70], (nq, 1)), np.tile([76, 129], (nq, 1))):
        want, mag = ref.attention(q64, k, v, scale, r)
        if r is not None and r is not ranges:
            assert np.isfinite(want).all()
        for many in forms(dtype):
            for ws in (True, False):
                with api.knobs(CACHE4_MANY=many):
                    o = attend(q, cache, cap, T, heads, d, scale, r, ws)
                close(o, want, mag, q64, k, scale, dtype, T, f"tokens that are no numbers, form {many}")


def test_attention_edges():
    heads, d, scale = 2, 64, 0.125
    # no tokens; no queries
    q, cache, cap, k, v = case(3, 7, 0, heads, d, "bf16")
    assert (attend(q, cache, cap, 0, heads, d, scale) == 0).all()
    assert (attend(q, cache, cap, 0, heads, d, scale, np.tile([0, 5], (7, 1))) == 0).all()
    o = torch.full((3, heads * d), 7.0, dtype=torch.bfloat16, device="cuda")
    api.sige_cache4_attn(o, cache, cap, o, scale, T=0, heads=heads, d=d, Nq=0)
    assert (o == 7.0).all()
    # logits of several hundred: the running maximum keeps the exponentials finite
    q, cache, cap, k, v = case(4, 70, 300, heads, d, "f16")
    q = (q * 30).contiguous()
    q64 = f64(q).reshape(-1, heads, d)
    want, mag = ref.attention(q64, k, v, scale)
    o = attend(q, cache, cap, 300, heads, d, scale)
    assert torch.isfinite(o).all()
    close(o, want, mag, q64, k, scale, "f16", 300, "large logits")
    # a scale of 0: the mean of the values
    o = attend(q, cache, cap, 300, heads, d, 0.0)
    close(o, np.broadcast_to(v.mean(0), want.shape), np.broadcast_to(np.abs(v).mean(0), want.shape), q64, k, 0.0, "f16", 300, "the mean")
    # queries of a row that are no numbers reach no other row
    q[3] = float("nan")
    q[4] = float("inf")
    got = attend(q, cache, cap, 300, heads, d, scale)
    keep = [i for i in range(70) if i not in (3, 4)]
    close(got[keep], want[keep], mag[keep], q64[keep], k, scale, "f16", 300, "beside rows of NaN")
    assert torch.isnan(got[3]).all()


@pytest.mark.parametrize("dtype,res,b,heads,d,n", [("bf16", 32, 8, 8, 40, 3), ("f16", 20, 8, 2, 24, 4), ("f32", 20, 4, 2, 64, 1)])
def test_attention_by_block_list(dtype, res, b, heads, d, n):
    """Queries read from a full tensor by block list: bit for bit the call that is handed those rows (pixels outside the map: the
    nearest inside it)."""
    C, T = heads * d, res * res
    full = rows(1, T, heads, d, dtype, ld=3 * C)
    _, cache, cap, _, _ = case(2, 1, T, heads, d, dtype)
    g = api.geom(res, res, b, 1, 1, 0)
    gx = -(-res // b)
    pick = np.sort(np.random.default_rng(d).permutation(gx * gx)[:n])
    pick[-1] = gx * gx - 1
    blocks = np.stack([pick // gx * b, pick % gx * b], 1).astype(np.int32)
    tok = [min(y0 + p // b, res - 1) * res + min(x0 + p % b, res - 1) for y0, x0 in blocks for p in range(b * b)]
    nq = n * b * b
    r = torch.from_numpy(some_ranges(nq, T, 3).astype(np.int32)).cuda()
    nb = api.sige_cache4_attn_workspace_bytes(nq, T, heads, d)
    w = torch.empty(max(nb // 4, 1), dtype=torch.float32, device="cuda")
    for ranges in (None, r):
        o = torch.full((nq + 1, C), 7.0, dtype=DT[dtype], device="cuda")
        api.sige_cache4_attn_blocks(full, g, torch.from_numpy(blocks).cuda(), n, cache, cap, o, 0.2, T=T, heads=heads, d=d,
                                    ranges=ranges, workspace=w)
        want = torch.full_like(o, 7.0)
        api.sige_cache4_attn(full[torch.tensor(tok, device="cuda")].contiguous(), cache, cap, want[:nq], 0.2, T=T, heads=heads, d=d,
                             ranges=ranges, workspace=w)
        torch.cuda.synchronize()
        assert torch.equal(o, want)


def test_attention_far_into_a_long_cache():
    """Tokens whose bytes lie more than 4 GiB into a section: stored, read back and seen."""
    heads, d, cap = 1, 256, 34_000_000
    n, nq = 90, 20
    cache = torch.empty(api.sige_cache4_bytes(heads, d, cap), dtype=torch.uint8, device="cuda")
    assert cache.numel() > 2 * 2 ** 32
    k, v = rows(1, n, heads, d, "bf16"), rows(2, n, heads, d, "bf16")
    first = cap - n
    api.sige_cache4_store(k, v, cache, cap, heads, d, first=first, n_rows=n)
    ko, vo = torch.empty_like(k), torch.empty_like(v)
    api.sige_cache4_load(cache, cap, heads, d, ko, vo, first=first)
    small = torch.empty(api.sige_cache4_bytes(heads, d, n), dtype=torch.uint8, device="cuda")
    api.sige_cache4_store(k, v, small, n, heads, d, n_rows=n)
    k2, v2 = torch.empty_like(k), torch.empty_like(v)
    api.sige_cache4_load(small, n, heads, d, k2, v2)
    torch.cuda.synchronize()
    assert torch.equal(ko, k2) and torch.equal(vo, v2)
    q = rows(3, nq, heads, d, "bf16")
    q64 = f64(q).reshape(nq, heads, d)
    k64, v64 = f64(k2).reshape(n, heads, d), f64(v2).reshape(n, heads, d)
    want, mag = ref.attention(q64, k64, v64, 0.0625)
    for ws in (False, True):
        o = attend(q, cache, cap, cap, heads, d, 0.0625, np.tile([first, cap], (nq, 1)), ws)
        close(o, want, mag, q64, k64, 0.0625, "bf16", n, "the last tokens of 34 million")


def test_attention_splits():
    """The keys cut over workgroups, as often as a workspace holds them (the knob aims for more and more workgroups)."""
    for dtype, nq, T, heads, d in (("bf16", 100, 3000, 1, 64), ("f16", 20, 5000, 2, 40), ("f32", 70, 2500, 1, 128), ("bf16", 150, 2000, 2, 96),
                                   ("f16", 40, 1500, 1, 200)):
        q, cache, cap, k, v = case(9, nq, T, heads, d, dtype)
        q64 = f64(q).reshape(nq, heads, d)
        scale = 1 / math.sqrt(d)
        ranges = some_ranges(nq, T, 8)
        for r in (None, ranges):
            want, mag = ref.attention(q64, k, v, scale, r)
            for many in forms(dtype):
                for wgs in (1, 3, 9, 40, 200):
                    with api.knobs(ATTN_WGS=wgs, CACHE4_MANY=many):
                        o = attend(q, cache, cap, T, heads, d, scale, r)
                    close(o, want, mag, q64, k, scale, dtype, T, f"form {many}, {wgs} workgroups")
        ws = torch.empty(3 * heads * nq * (d + 4), dtype=torch.float32, device="cuda")      # room for three
        o = torch.empty_like(q)
        api.sige_cache4_attn(q, cache, cap, o, scale, T=T, heads=heads, d=d, workspace=ws)
        want, mag = ref.attention(q64, k, v, scale)
        close(o, want, mag, q64, k, scale, dtype, T, "a small workspace")


def test_captured_and_on_another_stream():
    """Store and attention captured into a graph, replayed with new inputs between eager work; and on a stream of their own."""
    heads, d, T, nq = 8, 40, 1024, 48
    q, cache, cap, k, v = case(1, nq, T, heads, d, "bf16")
    kr, vr = rows(5, 16, heads, d, "bf16").clone(), rows(6, 16, heads, d, "bf16").clone()
    slots = torch.arange(100, 116, dtype=torch.int32, device="cuda")
    o = torch.empty_like(q)
    ws = torch.empty(api.sige_cache4_attn_workspace_bytes(nq, T, heads, d) // 4 + 1, dtype=torch.float32, device="cuda")

    def step():
        api.sige_cache4_store(kr, vr, cache, cap, heads, d, slots=slots, n_rows=16)
        api.sige_cache4_attn(q, cache, cap, o, 0.15, T=T, heads=heads, d=d, workspace=ws)

    step()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step()
    for i in range(4):
        kr.copy_(rows(20 + i, 16, heads, d, "bf16"))
        q.copy_(rows(30 + i, nq, heads, d, "bf16"))
        slots.add_(16)
        o.fill_(7.0)
        g.replay()
        got = o.clone()
        torch.cuda.synchronize()
        step()
        torch.cuda.synchronize()
        assert torch.equal(got, o), f"replay {i}"
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    want = o.clone()
    o.fill_(7.0)
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    side.synchronize()
    assert torch.equal(o, want)


def test_attention_takes_the_form_for_many_queries():
    """Calls that the rule gives to the forms for many queries (heads up to 64: more tiles of 32 queries than compute units; larger
    ones: tiles x tokens from 2^21 on), every row against float64 on the GPU."""
    for dtype, nq, T, heads, d in (("bf16", 2100, 300, 5, 64), ("f16", 1500, 700, 6, 40), ("bf16", 4200, 8200, 2, 96), ("f16", 4100, 16400, 1, 128)):
        q, cache, cap, k, v = case(7, nq, T, heads, d, dtype)
        k, v = torch.from_numpy(k).cuda(), torch.from_numpy(v).cuda()
        scale = 1 / math.sqrt(d)
        o = attend(q, cache, cap, T, heads, d, scale)
        q64 = q.double().view(nq, heads, d)
        for h in range(heads):
            s = q64[:, h] @ k[:, h].t() * scale
            p = torch.softmax(s, -1)
            want, mag = (p @ v[:, h]).cpu().numpy()[:, None], ((p + 2.0 ** -30) @ v[:, h].abs()).cpu().numpy()[:, None]
            close(o[:, h * d:(h + 1) * d], want, mag, q64[:, h:h + 1].cpu().numpy(), k[:, h:h + 1].cpu().numpy(), scale, dtype, T, f"{nq} of {T} x {d}")


def test_calls_at_once():
    """Two threads, each on a stream of its own with a workspace of its own, calling the same kernel for heads of two sizes: bit for bit
    what each call gives alone."""
    import threading
    jobs = []
    for d, T in ((72, 3000), (80, 900)):
        q, cache, cap, _, _ = case(d, 40, T, 3, d, "bf16")
        alone = attend(q, cache, cap, T, 3, d, 0.1).clone()
        ws = torch.empty(api.sige_cache4_attn_workspace_bytes(40, T, 3, d) // 4 + 1, dtype=torch.float32, device="cuda")
        jobs.append((q, cache, cap, T, d, alone, ws, [torch.empty(40, 3 * d, dtype=torch.bfloat16, device="cuda") for _ in range(20)]))
    torch.cuda.synchronize()
    errors = []

    def work(job):
        q, cache, cap, T, d, _, ws, outs = job
        try:
            with torch.cuda.stream(torch.cuda.Stream()):
                for o in outs:
                    api.sige_cache4_attn(q, cache, cap, o, 0.1, T=T, heads=3, d=d, workspace=ws)
        except Exception as e:                     # noqa: BLE001
            errors.append(e)
    threads = [threading.Thread(target=work, args=(j,)) for j in jobs]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    assert not errors, errors
    for _, _, _, _, _, alone, _, outs in jobs:
        assert all(torch.equal(o, alone) for o in outs)

"""What the rotary, 4-bit cache and adapter calls refuse, and what they compute on the host (no GPU: nothing below is enqueued)."""
import ctypes
import os

import numpy as np
import pytest
import torch

import cache4_oracle as ref
from paper_2211_02048_amd import api

FAKE = ctypes.c_void_p(0x10000)  # never dereferenced: every call below fails validation first
ODD = ctypes.c_void_p(0x10008)
F = ctypes.c_float(0.1)


@pytest.fixture(scope="module")
def L():
    if not os.path.exists(api.LIB_PATH):
        from paper_2211_02048_amd import build
        build.build()
    return api.lib()


def err(L):
    return L.sige_last_error().decode()


def good():
    return api.geom(16, 16, 4, 1, 1, 0)


def test_rope_pairs(L):
    t = api.sige_rope_pairs((3, 0, 5), 10000.0, device="cpu")
    f = t[:, 0].view(torch.float32).double() + t[:, 1].view(torch.float32).double()
    want = np.concatenate([10000.0 ** (-np.arange(3) / 3), 10000.0 ** (-np.arange(5) / 5)]) / (2 * np.pi)
    np.testing.assert_allclose(f.numpy(), want, rtol=2.0 ** -46)
    assert t[:, 2].tolist() == [0] * 3 + [2] * 5 and (t[:, 3] == 0).all()
    n = (ctypes.c_int32 * 2)(2, -1)
    assert L.sige_rope_pairs(n, 2, 10.0, FAKE) == 1 and "negative" in err(L)
    for theta in (0.0, -1.0, float("inf"), float("nan")):
        assert L.sige_rope_pairs((ctypes.c_int32 * 1)(2), 1, theta, FAKE) == 1
    assert L.sige_rope_pairs(None, 1, 10.0, FAKE) == 1
    assert L.sige_rope_pairs((ctypes.c_int32 * 1)(2), 0, 10.0, FAKE) == 1


def rope(L, x=FAKE, dt=1, heads=4, d=40, x_ld=160, count=None, per=0, mr=8, n=8, pairs=FAKE, n_pairs=20, layout=0, pos=FAKE, axes=2, y=FAKE, y_ld=160):
    return L.sige_token_rope(x, dt, heads, d, x_ld, count, per, mr, n, pairs, n_pairs, layout, pos, axes, y, y_ld, None)


def test_rope_refusals(L):
    assert rope(L, n=0) == 0 and err(L) == ""
    assert rope(L, x=None, n=0) == 0
    for kw in (dict(x=None), dict(y=None), dict(pairs=None), dict(pos=None), dict(dt=3), dict(heads=0), dict(d=0), dict(n_pairs=0), dict(n_pairs=21),
               dict(layout=2), dict(x_ld=152), dict(y_ld=152), dict(n=-1), dict(n=-1, count=FAKE), dict(n=-2), dict(mr=-1, n=-1, count=FAKE, per=1), dict(axes=0)):
        assert rope(L, **kw) == 1, kw
    for kw in (dict(d=36, x_ld=160, n_pairs=4), dict(x_ld=164), dict(y_ld=164), dict(x=ODD), dict(y=ODD), dict(pairs=ODD), dict(dt=0, x_ld=162)):
        assert rope(L, **kw) == 2, kw
    assert rope(L, n=9) == 3
    g = good()
    call = lambda g=g, idx=FAKE, count=FAKE, mb=4, n=2, axes=2: L.sige_token_rope_blocks(  # noqa: E731
        FAKE, 1, 4, 40, 160, ctypes.byref(g), idx, count, mb, n, FAKE, 20, 0, axes, F, FAKE, 160, None)
    assert call(n=0) == 0
    assert call(n=5) == 3 and call(idx=None) == 1 and call(count=None, n=-1) == 1 and call(axes=1) == 1 and call(axes=4) == 1
    assert call(g=api.geom(16, 16, 4, 3, 1, 1)) == 2


@pytest.mark.parametrize("d", [8, 16, 24, 32, 40, 64, 72, 80, 136, 160, 248, 256])
def test_cache_bytes(L, d):
    for heads, capacity in ((1, 1), (3, 32), (8, 33), (2, 100)):
        full, tail, gs = ref.sections(d)
        assert api.sige_cache4_bytes(heads, d, capacity) == heads * 2 * (-(-capacity // 32) * 32) * (16 * full + 8 * tail + gs)
    assert api.sige_cache4_bytes(8, d, 2 ** 31 - 1) == 16 * 2 ** 31 * sum(np.array(ref.sections(d)) * (16, 8, 1))


def test_cache_bytes_of_what_there_is_not(L):
    for heads, d, capacity in ((0, 64, 8), (1, 0, 8), (1, 64, 0), (1, 4, 8), (1, 12, 8), (1, 264, 8), (-1, 64, 8), (65536, 64, 8), (1, 64, -5)):
        assert api.sige_cache4_bytes(heads, d, capacity) == 0


def test_store_and_load_refusals(L):
    def store(k=FAKE, k_ld=320, v=FAKE, v_ld=320, dt=2, heads=8, d=40, slots=None, first=0, count=None, per=0, mr=8, n=8, cache=FAKE, cap=64):
        return L.sige_cache4_store(k, k_ld, v, v_ld, dt, heads, d, slots, first, count, per, mr, n, cache, cap, None)
    assert store(n=0) == 0
    for kw in (dict(k=None), dict(v=None), dict(cache=None), dict(dt=9), dict(heads=0), dict(d=0), dict(cap=0), dict(k_ld=312), dict(v_ld=312), dict(n=-1),
               dict(n=-1, count=FAKE), dict(first=-1), dict(slots=FAKE, first=1), dict(n=-2)):
        assert store(**kw) == 1, kw
    for kw in (dict(d=36), dict(d=264, heads=1), dict(k_ld=324), dict(v_ld=324), dict(k=ODD), dict(v=ODD), dict(cache=ODD), dict(dt=0, k_ld=322), dict(heads=70000)):
        assert store(**kw) == 2, kw
    assert store(n=9) == 3 and store(first=57) == 3 and "capacity" in err(L)

    def blocks(g=good(), idx=FAKE, count=FAKE, mb=4, n=2, first=0, cap=256):
        return L.sige_cache4_store_blocks(FAKE, 320, FAKE, 320, 2, 8, 40, ctypes.byref(g), idx, count, mb, n, first, FAKE, cap, None)
    assert blocks(n=0) == 0
    assert blocks(idx=None) == 1 and blocks(n=-1, count=None) == 1
    assert blocks(n=5) == 3 and blocks(cap=255) == 3 and blocks(first=1) == 3 and blocks(first=-1) == 3
    assert blocks(g=api.geom(16, 16, 4, 3, 1, 1)) == 2

    def load(cache=FAKE, cap=64, dt=1, heads=8, d=40, first=0, n=8, k=FAKE, k_ld=320, v=FAKE, v_ld=320):
        return L.sige_cache4_load(cache, cap, dt, heads, d, first, n, k, k_ld, v, v_ld, None)
    assert load(n=0) == 0
    for kw in (dict(cache=None), dict(k=None, v=None), dict(k_ld=312), dict(v_ld=312), dict(first=-1), dict(n=-1), dict(dt=-1)):
        assert load(**kw) == 1, kw
    assert load(k_ld=324) == 2 and load(v=ODD) == 2 and load(d=44) == 2
    assert load(n=65) == 3 and load(first=60) == 3 and load(first=2 ** 31 - 1, n=2 ** 31 - 1) == 3


def test_attention_refusals(L):
    def attn(q=FAKE, q_ld=320, cache=FAKE, cap=64, dt=2, nq=8, T=64, heads=8, d=40, scale=F, ranges=None, o=FAKE, o_ld=320):
        return L.sige_cache4_attn(q, q_ld, cache, cap, dt, nq, T, heads, d, scale, ranges, o, o_ld, None, 0, None)
    assert attn(nq=0, q=None, o=None) == 0
    for kw in (dict(q=None), dict(cache=None), dict(o=None), dict(dt=3), dict(nq=-1), dict(T=-1), dict(heads=0), dict(d=-8), dict(cap=0, T=0), dict(q_ld=312), dict(o_ld=312)):
        assert attn(**kw) == 1, kw
    for kw in (dict(d=36), dict(d=264, heads=1), dict(q_ld=324), dict(o_ld=324), dict(q=ODD), dict(o=ODD), dict(cache=ODD), dict(scale=ctypes.c_float(-1)),
               dict(scale=ctypes.c_float(float("nan"))), dict(heads=70000), dict(dt=0, q_ld=322)):
        assert attn(**kw) == 2, kw
    assert attn(T=65) == 3
    g = good()
    call = lambda g=g, idx=FAKE, n=2: L.sige_cache4_attn_blocks(FAKE, 320, ctypes.byref(g), idx, n, FAKE, 64, 2, 65 if n == 7 else 64, 8, 40, F, None, FAKE, 320, None, 0, None)  # noqa: E731
    assert call(n=0) == 0 and call(n=-1) == 1 and call(idx=None) == 1 and call(n=7) == 3 and call(g=api.geom(16, 16, 4, 3, 1, 1)) == 2
    for bad in ((0, 64, 8, 40), (8, 0, 8, 40), (8, 64, 0, 40), (8, 64, 8, 0), (8, 64, 8, 264)):
        assert api.sige_cache4_attn_workspace_bytes(*bad) == 0
    assert api.sige_cache4_attn_workspace_bytes(4, 65536, 1, 64) > 0


def test_lora_refusals(L):
    def lora(x=FAKE, dt=1, cin=320, x_ld=320, count=None, per=4, mr=8, n=8, down=FAKE, up=FAKE, rank=8, ad=2, alpha=None, ids=FAKE, base=FAKE, base_ld=64,
             cout=64, y=FAKE, y_ld=64):
        return L.sige_token_lora(x, dt, cin, x_ld, count, per, mr, n, down, up, rank, ad, alpha, ids, base, base_ld, cout, y, y_ld, None)
    assert lora(n=0) == 0
    for kw in (dict(x=None), dict(down=None), dict(up=None), dict(ids=None), dict(y=None), dict(dt=5), dict(cin=0), dict(cout=0), dict(rank=0), dict(ad=0), dict(per=0),
               dict(x_ld=312), dict(y_ld=56), dict(base_ld=56), dict(n=-1), dict(n=-2), dict(mr=-1, n=-1, count=FAKE)):
        assert lora(**kw) == 1, kw
    for kw in (dict(rank=136), dict(rank=12), dict(cin=324, x_ld=328), dict(cout=60), dict(x_ld=324), dict(y_ld=68), dict(base_ld=68), dict(x=ODD), dict(down=ODD),
               dict(up=ODD), dict(base=ODD), dict(y=ODD)):
        assert lora(**kw) == 2, kw
    assert lora(n=9) == 3
    assert lora(n=0, base=None, base_ld=0) == 0


def test_the_binding_refuses_what_it_can_see():
    """A cache tensor that is too small for the call, adapters of another shape, tensors that are not on the GPU."""
    q = torch.zeros(4, 128)
    small = torch.zeros(api.sige_cache4_bytes(2, 64, 32) - 1, dtype=torch.uint8)
    with pytest.raises(api.SigeError, match="takes"):
        api.sige_cache4_attn(q, small, 32, q, 1.0, T=4, heads=2, d=64)
    with pytest.raises(api.SigeError, match="takes"):
        api.sige_cache4_store(q, q, small, 32, 2, 64, n_rows=4)
    with pytest.raises(api.SigeError, match="contiguous"):
        api.sige_token_lora(q, q, 128, 128, torch.zeros(2, 8, 128), torch.zeros(2, 8, 128), None, 4, n_rows=4)


def test_more_than_a_launch_can_have(L):
    """Calls of more threads than a launch has, aliases whose rows lie at other distances, tokens whose chunks would end past an int."""
    big = 2 ** 31 - 1
    assert rope(L, mr=big, n=big) == 2
    assert rope(L, y=FAKE, y_ld=168) == 2 and "stride" in err(L)
    assert L.sige_cache4_store(FAKE, 320, FAKE, 320, 2, 8, 40, None, 0, None, 0, 2 ** 27, 2 ** 27, FAKE, 2 ** 27, None) == 2 and "rows" in err(L)
    assert L.sige_cache4_load(FAKE, 2 ** 27, 2, 8, 40, 0, 2 ** 27, FAKE, 320, FAKE, 320, None) == 2
    assert L.sige_cache4_attn(FAKE, 320, FAKE, big, 2, 8, big, 8, 40, F, None, FAKE, 320, None, 0, None) == 2 and "tokens" in err(L)
    for dt, d in ((2, 40), (1, 128), (0, 256)):
        assert L.sige_cache4_attn(FAKE, 8 * d, FAKE, 64, dt, big, 64, 8, d, F, None, FAKE, 8 * d, None, 0, None) == 2 and "queries" in err(L)
    other = ctypes.c_void_p(0x20000)
    lora = lambda n=8, y=other, base=None, base_ld=64, y_ld=64: L.sige_token_lora(  # noqa: E731
        FAKE, 1, 320, 320, None, 4, n, n, FAKE, FAKE, 8, 2, None, FAKE, base, base_ld, 64, y, y_ld, None)
    assert lora(y=FAKE) == 2 and "y cannot be x" in err(L)
    assert lora(base=other, y_ld=72) == 2 and "stride" in err(L)
    assert lora(n=2 ** 28) == 2 and "rows" in err(L)


def test_the_binding_refuses_tables_and_types():
    """Tables of another type or too short (ids of 64 bits, ranges of fewer rows), operands of different types."""
    h, i = torch.bfloat16, torch.int32
    x = torch.zeros(8, 128, dtype=h)
    cache = torch.zeros(api.sige_cache4_bytes(2, 64, 32), dtype=torch.uint8)
    table = torch.zeros(32, 4, dtype=i)
    g = good()
    idx, cnt = torch.zeros(2, 2, dtype=i), torch.zeros(1, dtype=i)
    down, up = torch.zeros(2, 8, 128, dtype=h), torch.zeros(2, 128, 8, dtype=h)
    calls = {
        "bfloat16": [lambda: api.sige_token_rope(x, x.float(), 2, 64, table, torch.zeros(8, 2), n_rows=8),
                     lambda: api.sige_cache4_store(x, x.float(), cache, 32, 2, 64, n_rows=8),
                     lambda: api.sige_cache4_load(cache, 32, 2, 64, x, x.half()),
                     lambda: api.sige_cache4_attn(x, cache, 32, x.float(), 1.0, T=4, heads=2, d=64),
                     lambda: api.sige_token_lora(x, x, 128, 128, down.float(), up, torch.zeros(2, dtype=i), 4, n_rows=8),
                     lambda: api.sige_token_lora(x, x, 128, 128, down, up, torch.zeros(2, dtype=i), 4, base=x.float(), n_rows=8)],
        "pairs": [lambda: api.sige_token_rope(x, x, 2, 64, table.long(), torch.zeros(8, 2), n_rows=8)],
        "positions": [lambda: api.sige_token_rope(x, x, 2, 64, table, torch.zeros(8, 2, dtype=torch.float64), n_rows=8),
                      lambda: api.sige_token_rope(x, x, 2, 64, table, torch.zeros(7, 2), n_rows=8),
                      lambda: api.sige_token_rope(x, x, 2, 64, table, torch.zeros(2, 8).t(), n_rows=8)],
        "indices": [lambda: api.sige_token_rope_blocks(x, x, 2, 64, table, g, idx.long(), cnt),
                    lambda: api.sige_cache4_store_blocks(x, x, cache, 32, 2, 64, g, idx, cnt, n_blocks=3),
                    lambda: api.sige_cache4_attn_blocks(x, g, idx, 3, cache, 32, x, 1.0, T=4, heads=2, d=64)],
        "count": [lambda: api.sige_token_rope_blocks(x, x, 2, 64, table, g, idx, cnt.long())],
        "slots": [lambda: api.sige_cache4_store(x, x, cache, 32, 2, 64, slots=torch.zeros(8, dtype=torch.int64), n_rows=8),
                  lambda: api.sige_cache4_store(x, x, cache, 32, 2, 64, slots=torch.zeros(7, dtype=i), n_rows=8)],
        "ranges": [lambda: api.sige_cache4_attn(x, cache, 32, x, 1.0, T=4, heads=2, d=64, ranges=torch.zeros(7, 2, dtype=i)),
                   lambda: api.sige_cache4_attn(x, cache, 32, x, 1.0, T=4, heads=2, d=64, ranges=torch.zeros(8, 2)),
                   lambda: api.sige_cache4_attn_blocks(x, g, idx, 2, cache, 32, x, 1.0, T=4, heads=2, d=64, ranges=torch.zeros(31, 2, dtype=i))],
        "ids": [lambda: api.sige_token_lora(x, x, 128, 128, down, up, torch.zeros(2, dtype=torch.int64), 4, n_rows=8),
                lambda: api.sige_token_lora(x, x, 128, 128, down, up, torch.zeros(2, dtype=i), 3, n_rows=8)],
        "alpha": [lambda: api.sige_token_lora(x, x, 128, 128, down, up, torch.zeros(2, dtype=i), 4, alpha=torch.zeros(1), n_rows=8)],
    }
    for what, bad in calls.items():
        for call in bad:
            with pytest.raises(api.SigeError, match=what):
                call()


def test_the_binding_refuses_gaps_between_rows():
    """Tiles of 1 x 8 pixels out of tiles of 1 x 10: the rows do not follow each other at one distance, whatever the axis of one says;
    an axis of one between rows that do is no gap."""
    h, i = torch.bfloat16, torch.int32
    wide, y = torch.zeros(4, 1, 10, 128, dtype=h), torch.zeros(40, 128, dtype=h)
    down, up, ids = torch.zeros(2, 8, 128, dtype=h), torch.zeros(2, 128, 8, dtype=h), torch.zeros(10, dtype=i)
    for x, n, what in ((wide[:, :, :8], 32, "one distance"), (wide, 40, "cpu"), (wide[:, :, :, :64], 40, "cpu"),
                       (torch.zeros(4, 3, 10, 128, dtype=h)[:, :1], 40, "one distance"), (torch.zeros(4, 3, 128, dtype=h)[:, :1], 4, "cpu")):
        c = x.shape[-1]
        with pytest.raises(api.SigeError, match=what):
            api.sige_token_lora(x, y, c, 128, down[:, :, :c].contiguous(), up, ids, 4, n_rows=n)


def test_the_binding_refuses_rows_that_are_not_there():
    """Tensors with fewer rows or channels than the call touches, rows given by a stride of the caller's that pass the storage's end,
    rows with gaps between them; the whole ones get as far as the refusal of CPU tensors."""
    h, i = torch.bfloat16, torch.int32
    R, C = 32, 128
    x, y = torch.zeros(R, C, dtype=h), torch.zeros(R, C, dtype=h)
    short, narrow, flat, small = x[:R - 1], x[:, :C - 8], torch.zeros(R * C, dtype=h), torch.zeros(R * C - 1, dtype=h)
    cache = torch.zeros(api.sige_cache4_bytes(2, 64, 256), dtype=torch.uint8)
    table, pos = torch.zeros(32, 4, dtype=i), torch.zeros(R, 2)
    g = good()                                            # 16 x 16 pixels, blocks of 4 x 4
    idx, cnt = torch.zeros(2, 2, dtype=i), torch.zeros(1, dtype=i)
    full = torch.zeros(256, C, dtype=h)
    down, up, ids = torch.zeros(2, 8, C, dtype=h), torch.zeros(2, C, 8, dtype=h), torch.zeros(8, dtype=i)

    def rope(a, b, n=R, **kw):
        return lambda: api.sige_token_rope(a, b, 2, 64, table, pos, n_rows=n, **{"max_rows": R, **kw})

    def rope_blocks(a, b, n=2):
        return lambda: api.sige_token_rope_blocks(a, b, 2, 64, table, g, idx, cnt, n_blocks=n)

    def store(k, v, **kw):
        return lambda: api.sige_cache4_store(k, v, cache, 256, 2, 64, **{"n_rows": R, "max_rows": R, **kw})

    def store_blocks(k, v, n=2):
        return lambda: api.sige_cache4_store_blocks(k, v, cache, 256, 2, 64, g, idx, cnt, n_blocks=n)

    def load(k, v, **kw):
        return lambda: api.sige_cache4_load(cache, 256, 2, 64, k, v, **kw)

    def attn(q, o, **kw):
        return lambda: api.sige_cache4_attn(q, cache, 256, o, 1.0, T=4, heads=2, d=64, **kw)

    def attn_blocks(q, o):
        return lambda: api.sige_cache4_attn_blocks(q, g, idx, 2, cache, 256, o, 1.0, T=4, heads=2, d=64)

    def lora(a, b, base=None, **kw):
        return lambda: api.sige_token_lora(a, b, C, C, down, up, ids, 4, base=base, **{"n_rows": R, "max_rows": R, **kw})

    tiles = torch.zeros(4, 1, 10, C, dtype=h)             # rows of a tile of 1 x 8 out of tiles of 1 x 10
    whole = [rope(x, y), rope(x, x), rope(flat, y, x_ld=C), rope(x.view(2, 4, 4, C), y), rope(short, y, n=R - 1), rope_blocks(x, y), rope_blocks(x, y, -1),
             rope_blocks(short, short, 1), store(x, y), store(x.view(R, 2, 64), flat, v_ld=C), store(short, y, n_rows=-1, max_rows=R - 1, count=cnt, rows_per_count=4),
             store_blocks(x, y), load(x, y), load(None, y), load(short, y), load(x, flat, v_ld=C), attn(x, y), attn(short, y), attn(x, flat, o_ld=C),
             attn(x.view(R, 2, 64), y), attn_blocks(full, y), attn_blocks(full.view(16, 16, C), y), lora(x, y), lora(x, y, x), lora(x, flat, y_ld=C),
             lora(x.view(8, 2, 2, C), y), lora(x.view(8, 1, 4, C), y), lora(tiles[:2, :, :, :], y, n_rows=20), lora(short, short, n_rows=R - 1),
             attn(x, y, Nq=0), rope(x, y[:0], n=0)]
    for call in whole:
        with pytest.raises(api.SigeError, match="cpu"):
            call()
    missing = [rope(short, y), rope(x, short), rope(narrow, y), rope(x, narrow), rope(x, small, y_ld=C), rope(x, y, x_ld=C + 8), rope(x[1:], y, x_ld=C),
               rope(x, short, n=-1, count=cnt, rows_per_count=4), rope(x.view(2, 16, C)[:, :15], y), rope_blocks(short, y), rope_blocks(x, short), rope_blocks(short, y, -1),
               store(short, y), store(x, short), store(x, narrow), store(x, short, n_rows=-1, count=cnt, rows_per_count=4), store(x, flat[8:], v_ld=C),
               store(x, x.view(R, 2, 64)[:R - 1]), store_blocks(x, short), store_blocks(short, y), store_blocks(x, short, -1),
               load(x, short), load(short, y, n_tokens=R), load(x, narrow), load(x, y, n_tokens=R + 1), load(x, flat, v_ld=C + 8),
               attn(x, short), attn(short, y, Nq=R), attn(x, narrow), attn(x, small, o_ld=C), attn_blocks(full[:255], y), attn_blocks(full, short),
               attn_blocks(full[:, :120], y), lora(x, short), lora(short, y), lora(x, y, short), lora(x, narrow), lora(narrow, y), lora(x, y, narrow),
               lora(x, flat[1:], y_ld=C), lora(x, y, flat[8:], base_ld=C), lora(tiles[:, :, :8], y), lora(x, y[:1].expand(R, C)[:R - 1])]
    for call in missing:
        with pytest.raises(api.SigeError, match="rows of"):
            call()
    for call, what in ((load(None, None), "k or v"), (lambda: api.sige_cache4_attn(x, cache.expand(2, -1), 256, y, 1.0, T=4, heads=2, d=64), "contiguous"),
                       (lambda: api.sige_cache4_attn(x, cache, 256, y, 1.0, T=4, heads=2, d=64, workspace=torch.zeros(1).expand(4096)), "contiguous"),
                       (lambda: api.sige_token_rope_blocks(x, y, 2, 64, table, g, idx, cnt[:0]), "count")):
        with pytest.raises(api.SigeError, match=what):
            call()


def test_adapters_of_more_channels_than_offsets_count(L):
    for cin, cout in ((320, 2 ** 30 + 8), (320, 2 ** 31 - 8), (2 ** 30, 64), (320, 2 ** 28 + 8)):
        for dt in (0, 1):
            assert L.sige_token_lora(FAKE, dt, cin, cin, None, 4, 8, 8, FAKE, FAKE, 8, 2, None, FAKE, None, 0, cout, ctypes.c_void_p(0x20000), cout, None) == 2
            assert "channels" in err(L)

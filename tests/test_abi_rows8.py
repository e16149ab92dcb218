"""What the calls for rows in 8 bits refuse, and the oracle's own conversions (no GPU: nothing below is enqueued)."""
import ctypes
import os

import numpy as np
import pytest
import torch

import rows8_oracle as ref
from paper_2211_02048_amd import api

FAKE = ctypes.c_void_p(0x10000)  # never dereferenced: every call below fails validation first
OTHER = ctypes.c_void_p(0x20000)
ODD = ctypes.c_void_p(0x10008)
ODDER = ctypes.c_void_p(0x10002)


@pytest.fixture(scope="module")
def L():
    if not os.path.exists(api.LIB_PATH):
        from paper_2211_02048_amd import build
        build.build()
    return api.lib()


def err(L):
    return L.sige_last_error().decode()


def test_oracle_conversion_against_torch():
    """The oracle's codes are those of torch's cast to the type."""
    rng = np.random.default_rng(0)
    x = np.concatenate([rng.normal(size=4096) * 2.0 ** rng.integers(-12, 8, 4096), ref.MAG, -ref.MAG, ref.EDGES, -ref.EDGES, [0.0, -0.0]])
    x = x[np.abs(x) <= 448].astype(np.float32)
    want = torch.from_numpy(x).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    got = ref.nearest_code(np.abs(x).astype(float)) | np.where(np.signbit(x), 0x80, 0).astype(np.uint8)
    np.testing.assert_array_equal(got, want)
    x = rng.normal(size=(5, 300)) * np.exp(3 * rng.normal(size=(5, 1)))
    q, s = ref.store(x)
    v = ref.values(q, s, 300)
    top = np.abs(np.pad(x, ((0, 0), (0, 84)))).reshape(5, 3, 128).max(-1)
    scale = 2.0 ** (s[:, :3].astype(float) - 127)
    assert (top <= 448 * scale).all() and (top > 224 * scale).all() and (s[:, 3:] == 0).all() and (q[:, 300:] == 0).all()
    assert (np.abs(v - x) <= 2.0 ** -4 * np.abs(x) + 2.0 ** -10 * np.repeat(scale, 128, 1)[:, :300]).all()


def test_sizes():
    for C, want in ((1, (128, 4)), (128, (128, 4)), (129, (256, 4)), (512, (512, 4)), (513, (640, 8)), (1288, (1408, 12))):
        assert api.rows8_lds(C) == want == ref.lds(C)


def test_store_and_load_refusals(L):
    def store(x=FAKE, dt=1, C=320, x_ld=320, count=None, per=0, mr=8, n=8, q=FAKE, q_ld=384, s=FAKE, s_ld=4):
        return L.sige_rows8_store(x, dt, C, x_ld, count, per, mr, n, q, q_ld, s, s_ld, None)

    def load(x=FAKE, dt=1, C=320, x_ld=320, count=None, per=0, mr=8, n=8, q=FAKE, q_ld=384, s=FAKE, s_ld=4):
        return L.sige_rows8_load(q, q_ld, s, s_ld, C, count, per, mr, n, x, dt, x_ld, None)
    for call in (store, load):
        assert call(n=0) == 0 and err(L) == ""
        assert call(n=0, x=None, q=None, s=None) == 0
        for kw in (dict(x=None), dict(q=None), dict(s=None), dict(dt=3), dict(C=0), dict(C=-8), dict(x_ld=312), dict(q_ld=368), dict(s_ld=0), dict(C=520, x_ld=520, q_ld=640),
                   dict(n=-1), dict(n=-1, count=FAKE), dict(n=-2), dict(mr=-1, n=-1, count=FAKE, per=1)):
            assert call(**kw) == 1, kw
        for kw in (dict(C=316, x_ld=320), dict(x_ld=324), dict(x=ODD), dict(q=ODD), dict(s=ODDER), dict(q_ld=392), dict(s_ld=6), dict(dt=0, x_ld=322),
                   dict(mr=2 ** 31 - 1, n=2 ** 31 - 1), dict(mr=2 ** 26, n=2 ** 26), dict(mr=2 ** 26, n=-1, count=FAKE, per=1), dict(C=520, x_ld=520, q_ld=640, s_ld=8, mr=2 ** 25, n=2 ** 25)):
            assert call(**kw) == 2, kw
        assert call(n=9) == 3


def test_rms_refusals(L):
    def rms(x=FAKE, dt=1, C=320, x_ld=320, res=None, res_ld=0, count=None, per=0, mr=8, n=8, gamma=None, eps=1e-6, total=None, total_ld=0, y=OTHER, y_ld=320,
            q=None, q_ld=0, s=None, s_ld=0):
        return L.sige_token_rms(x, dt, C, x_ld, res, res_ld, count, per, mr, n, gamma, ctypes.c_float(eps), total, total_ld, y, y_ld, q, q_ld, s, s_ld, None)
    assert rms(n=0) == 0 and err(L) == ""
    for kw in (dict(x=None), dict(y=None), dict(dt=3), dict(C=0), dict(x_ld=312), dict(y_ld=312), dict(res=FAKE, res_ld=312), dict(total=FAKE, total_ld=320),
               dict(res=FAKE, res_ld=320, total=FAKE, total_ld=312), dict(q=FAKE, q_ld=368, s=FAKE, s_ld=4), dict(q=FAKE, q_ld=384, s=None, s_ld=4),
               dict(eps=-1.0), dict(eps=float("nan")), dict(n=-1), dict(n=-2), dict(res=FAKE, res_ld=320, total=OTHER, total_ld=320)):
        assert rms(**kw) == 1, kw
    for kw in (dict(C=316), dict(x=ODD), dict(y=ODD), dict(res=ODD, res_ld=320), dict(gamma=ODDER), dict(C=16392, x_ld=16392, y_ld=16392), dict(y=FAKE, y_ld=328),
               dict(q=ODD, q_ld=384, s=FAKE, s_ld=4), dict(res=FAKE, res_ld=320, total=FAKE, total_ld=328), dict(res=OTHER, res_ld=328, total=OTHER, total_ld=320, y=None, q=FAKE, q_ld=384, s=FAKE, s_ld=4),
               dict(dt=0, C=8196, x_ld=8196, y_ld=8196), dict(mr=2 ** 26, n=2 ** 26)):
        assert rms(**kw) == 2, kw
    assert rms(n=9) == 3


def test_rms_more_workgroups_than_a_launch_has(L):
    # single precision, three chunks of 512 channels: a workgroup of 256 threads per row, and a launch has fewer than 2^32 threads (four
    # chunks: the limit of 2^26 rows times chunks comes first)
    n = 2 ** 24
    for C in (1028, 1536):
        assert L.sige_token_rms(FAKE, 0, C, C, None, 0, None, 0, n, n, None, ctypes.c_float(1e-6), None, 0, OTHER, C, None, 0, None, 0, None) == 2
        assert "2^24" in err(L)


def test_8_bit_rows_in_the_place_of_others_are_refused(L):
    THIRD = ctypes.c_void_p(0x30000)
    assert L.sige_rows8_store(FAKE, 1, 512, 512, None, 0, 8, 8, FAKE, 512, OTHER, 4, None) == 1 and "place" in err(L)
    assert L.sige_rows8_store(FAKE, 1, 512, 512, None, 0, 8, 8, OTHER, 512, FAKE, 4, None) == 1
    assert L.sige_rows8_store(FAKE, 1, 512, 512, None, 0, 8, 8, OTHER, 512, OTHER, 4, None) == 1
    assert L.sige_rows8_load(FAKE, 512, OTHER, 4, 512, None, 0, 8, 8, FAKE, 1, 512, None) == 1 and "place" in err(L)
    assert L.sige_rows8_load(FAKE, 512, OTHER, 4, 512, None, 0, 8, 8, OTHER, 1, 512, None) == 1

    def rms(q, s, x=FAKE, res=None, total=None, y=None):
        return L.sige_token_rms(x, 1, 512, 512, res, 512, None, 0, 8, 8, None, ctypes.c_float(1e-6), total, 512, y, 512, q, 512, s, 4, None)
    FOURTH = ctypes.c_void_p(0x40000)
    for kw in (dict(q=FAKE, s=FOURTH), dict(q=FOURTH, s=FAKE), dict(q=FOURTH, s=FOURTH), dict(q=OTHER, s=FOURTH, res=OTHER), dict(q=OTHER, s=FOURTH, y=OTHER),
               dict(q=FOURTH, s=OTHER, y=OTHER), dict(q=THIRD, s=FOURTH, res=OTHER, total=THIRD), dict(q=FOURTH, s=THIRD, res=OTHER, total=THIRD)):
        assert rms(**kw) == 1 and "place" in err(L), kw


def test_linear_refusals(L):
    def linear(x=FAKE, x_ld=384, xs=FAKE, xs_ld=4, cin=320, count=None, per=0, mr=8, n=8, w=FAKE, w_ld=384, ws=FAKE, ws_ld=4, cout=640, bias=None, base=None, base_ld=0,
               y=OTHER, dt=1, y_ld=640):
        return L.sige_rows8_linear(x, x_ld, xs, xs_ld, cin, count, per, mr, n, w, w_ld, ws, ws_ld, cout, bias, base, base_ld, y, dt, y_ld, None)

    def gated(x=FAKE, x_ld=384, xs=FAKE, xs_ld=4, cin=320, count=None, per=0, mr=8, n=8, w=FAKE, w_ld=384, ws=FAKE, ws_ld=4, cout=640, bias=None, gate=0, q=OTHER, q_ld=640,
              s=OTHER, s_ld=8):
        return L.sige_rows8_linear_gated(x, x_ld, xs, xs_ld, cin, count, per, mr, n, w, w_ld, ws, ws_ld, cout, bias, gate, q, q_ld, s, s_ld, None)
    for call in (linear, gated):
        assert call(n=0) == 0 and err(L) == ""
        for kw in (dict(x=None), dict(xs=None), dict(w=None), dict(ws=None), dict(cin=0), dict(cout=0), dict(x_ld=368), dict(w_ld=368), dict(xs_ld=0), dict(cin=520, x_ld=640, w_ld=640, ws_ld=8),
                   dict(n=-1), dict(n=-1, count=FAKE), dict(n=-2)):
            assert call(**kw) == 1, kw
        for kw in (dict(x=ODD), dict(w=ODD), dict(xs=ODDER), dict(ws=ODDER), dict(x_ld=392), dict(w_ld=392), dict(xs_ld=6), dict(ws_ld=6), dict(cout=636), dict(bias=ODDER),
                   dict(cout=2 ** 28 + 8, y_ld=2 ** 29) if call is linear else dict(cout=2 ** 28 + 8, q_ld=2 ** 29, s_ld=2 ** 24)):
            assert call(**kw) == 2, kw
        assert call(n=9) == 3
    for kw in (dict(y=None), dict(dt=3), dict(y_ld=632), dict(base=FAKE, base_ld=632), dict(y=FAKE)):
        assert linear(**kw) == 1, kw
    for form, dt in ((8, 1), (7, 0), (100, 2)):
        with api.knobs(ROWS8_FORM=form):
            assert linear(dt=dt) == 2 and "form" in err(L)
            assert form == 7 or gated() == 2
    for kw in (dict(y=ODD), dict(base=ODD, base_ld=640), dict(y_ld=644), dict(base=OTHER, base_ld=648), dict(dt=0, cout=642, y_ld=644)):
        assert linear(**kw) == 2, kw
    for kw in (dict(gate=2), dict(gate=-1), dict(q=None), dict(s=None), dict(q_ld=624), dict(s_ld=4), dict(q=FAKE), dict(s=FAKE)):
        assert gated(**kw) == 1, kw
    for kw in (dict(q=ODD), dict(s=ODDER), dict(q_ld=648), dict(s_ld=10)):
        assert gated(**kw) == 2, kw


def test_binding_refusals():
    """What the binding refuses before it asks the library."""
    x, y = torch.zeros(4, 320, dtype=torch.float16), torch.zeros(4, 640, dtype=torch.float16)
    q, s = api.rows8(4, 320, "cpu")
    w, ws = api.rows8(640, 320, "cpu")
    o, os_ = api.rows8(4, 640, "cpu")

    def refused(code, fn, *a, **kw):
        with pytest.raises(api.SigeError) as e:
            fn(*a, **kw)
        assert e.value.code == code, e.value
    refused(1, api.sige_rows8_store, x, q, s, 320, n_rows=4)                                       # on the CPU
    refused(1, api.sige_rows8_store, x, q.char(), s, 320, n_rows=4)
    refused(3, api.sige_rows8_store, x, q[:3], s, 320, n_rows=4)
    refused(3, api.sige_rows8_store, x, q[:, :368], s, 320, n_rows=4)
    refused(3, api.sige_rows8_store, x, q, s[:, :3], 320, n_rows=4)
    refused(1, api.sige_rows8_store, x, q.t().contiguous().t(), s, 320, n_rows=4)
    refused(3, api.sige_rows8_store, x, q, s, 320, n_rows=5)
    refused(1, api.sige_rows8_store, x, q.flatten(), s, 320, n_rows=4)
    refused(1, api.sige_rows8_load, q, s.view(2, 2, 4), x, 320, n_rows=4)
    refused(3, api.sige_rows8_store, x, q, s, 328, n_rows=4)
    refused(3, api.sige_rows8_load, q, s, x[:, :312], 320, n_rows=4)
    refused(1, api.sige_token_rms, x, 320, torch.ones(320, dtype=torch.float16), y=x, n_rows=4)
    refused(1, api.sige_token_rms, x, 320, torch.ones(312), y=x, n_rows=4)
    refused(1, api.sige_token_rms, x, 320, y=x.float(), n_rows=4)
    refused(1, api.sige_token_rms, x, 320, q=q, n_rows=4)
    refused(3, api.sige_token_rms, x, 320, q=q, scales=s[:3], n_rows=4)
    refused(3, api.sige_token_rms, x, 320, y=x, residual=x[:3], n_rows=4)
    refused(1, api.sige_rows8_linear, q, s, w, ws, y, 320, 640, bias=torch.zeros(632), n_rows=4)
    refused(1, api.sige_rows8_linear, q, s, w, ws, y, 320, 640, base=y.float(), n_rows=4)
    refused(3, api.sige_rows8_linear, q, s, w[:639], ws, y, 320, 640, n_rows=4)
    refused(3, api.sige_rows8_linear, q[:3], s, w, ws, y, 320, 640, n_rows=4)
    refused(3, api.sige_rows8_linear, q, s, w, ws, y, 520, 640, n_rows=4)
    refused(3, api.sige_rows8_linear_gated, q, s, w, ws, o, os_, 320, 640, n_rows=4)               # 2 * 640 rows of weights
    refused(3, api.sige_rows8_linear_gated, q, s, w, ws, o[:, :304], os_, 320, 320, n_rows=4)
    refused(1, api.sige_rows8_linear_gated, q, s, w, ws, o, os_, 320, 320, bias=torch.zeros(320), n_rows=4)
    refused(1, api.sige_rows8_linear_gated, q, s, w, ws, o, os_, 320, 320, n_rows=-1, count=torch.zeros(1), rows_per_count=1)


def test_limits_at_the_end_of_32_bits(L):
    """Rounding up to a tile's rows or a chunk's channels has to stay a positive number: no form's launch holds these calls."""
    n = 2 ** 31 - 1
    THIRD, FOURTH = ctypes.c_void_p(0x30000), ctypes.c_void_p(0x40000)
    for rows in (n, n - 14, n - 127, n - 254):
        for count, per, host in ((None, 0, rows), (FAKE, 1, -1)):
            for form in range(-1, 8):
                with api.knobs(ROWS8_FORM=form):
                    for dt in (0, 1, 2) if form < 7 else (1, 2):
                        assert L.sige_rows8_linear(FAKE, 384, FAKE, 4, 320, count, per, rows, host, FAKE, 384, FAKE, 4, 640, None, None, 0, OTHER, dt, 640, None) == 2, (rows, form, dt)
                    if form < 4:
                        assert L.sige_rows8_linear_gated(FAKE, 384, FAKE, 4, 320, count, per, rows, host, FAKE, 384, FAKE, 4, 640, None, 0, THIRD, 640, FOURTH, 8, None) == 2, (rows, form)
            assert L.sige_token_rms(FAKE, 1, 320, 320, None, 0, count, per, rows, host, None, ctypes.c_float(1e-6), None, 0, OTHER, 320, None, 0, None, 0, None) == 2
    # sixteen rows of 2^31 - 128 channels are 2^26 times 512 channels begun, and so many channels and 511 more do not fit an int
    for C in (2 ** 31 - 128, 2 ** 31 - 504):
        ld = -(-C // 128) * 128
        assert L.sige_rows8_store(FAKE, 1, C, C, None, 0, 16, 16, THIRD, ld, FOURTH, 2 ** 24, None) == 2
        assert L.sige_rows8_load(FAKE, ld, OTHER, 2 ** 24, C, None, 0, 16, 16, THIRD, 1, C, None) == 2


def test_a_launch_has_fewer_than_2_32_threads(L):
    """Four waves of 64 make a workgroup: from 2^26 - 3 waves on there would be 2^24 workgroups of 256 threads."""
    THIRD, FOURTH = ctypes.c_void_p(0x30000), ctypes.c_void_p(0x40000)
    for n in (2 ** 26 - 3, 2 ** 26 - 2, 2 ** 26 - 1):
        for count, per, host in ((None, 0, n), (FAKE, 1, -1)):
            for C in (8, 512):
                assert L.sige_rows8_store(FAKE, 1, C, C, count, per, n, host, THIRD, 512, FOURTH, 4, None) == 2 and "2^26" in err(L)
                assert L.sige_rows8_load(THIRD, 512, FOURTH, 4, C, count, per, n, host, FAKE, 1, C, None) == 2
                assert L.sige_token_rms(FAKE, 1, C, C, None, 0, count, per, n, host, None, ctypes.c_float(1e-6), None, 0, OTHER, C, None, 0, None, 0, None) == 2


def test_outputs_in_the_place_of_other_tensors_are_refused(L):
    """Products: a tensor that another workgroup still reads, or that another output is written to."""
    at = {name: ctypes.c_void_p(0x100000 * (i + 1)) for i, name in enumerate(("x", "xs", "w", "ws", "bias", "base", "y", "q", "s", "gamma"))}

    def linear(**kw):
        p = {**at, **kw}
        return L.sige_rows8_linear(p["x"], 512, p["xs"], 4, 512, None, 0, 8, 8, p["w"], 512, p["ws"], 4, 512, p["bias"], p["base"], 512, p["y"], 1, 512, None)

    def gated(**kw):
        p = {**at, **kw}
        return L.sige_rows8_linear_gated(p["x"], 512, p["xs"], 4, 512, None, 0, 8, 8, p["w"], 512, p["ws"], 4, 512, p["bias"], 0, p["q"], 512, p["s"], 4, None)

    def rms(**kw):
        p = {**at, **kw}
        return L.sige_token_rms(p["x"], 1, 512, 512, p["base"], 512, None, 0, 8, 8, p["gamma"], ctypes.c_float(1e-6), p["w"], 512, p["y"], 512, p["q"], 512, p["s"], 4, None)
    for name in ("x", "xs", "w", "ws", "bias"):
        assert linear(y=at[name]) == 1 and "place" in err(L), name
        assert gated(q=at[name]) == 1 and "place" in err(L), name
        assert gated(s=at[name]) == 1 and "place" in err(L), name
    assert gated(s=at["q"]) == 1 and "place" in err(L)
    for out in ("w", "y", "q", "s"):                            # (w: the sum)
        assert rms(**{out: at["gamma"]}) == 1 and "place" in err(L), out
    # calls without rows touch nothing
    assert L.sige_rows8_linear_gated(at["x"], 512, at["xs"], 4, 512, None, 0, 8, 0, at["w"], 512, at["ws"], 4, 512, None, 0, at["q"], 512, at["q"], 4, None) == 0


def test_calls_without_rows_take_tensors_without_memory(L):
    """An edit that touches nothing: tensors of no rows, whose addresses are null."""
    eps = ctypes.c_float(1e-6)
    for count, per, mr, host in ((None, 0, 0, 0), (FAKE, 16, 0, -1), (None, 0, 8, 0)):
        rows = (count, per, mr, host)
        assert L.sige_rows8_store(None, 1, 320, 320, *rows, None, 384, None, 4, None) == 0
        assert L.sige_rows8_load(None, 384, None, 4, 320, *rows, None, 1, 320, None) == 0
        assert L.sige_rows8_linear(None, 384, None, 4, 320, *rows, FAKE, 384, FAKE, 4, 640, None, None, 0, None, 1, 640, None) == 0
        assert L.sige_rows8_linear_gated(None, 384, None, 4, 320, *rows, FAKE, 384, FAKE, 4, 640, None, 0, None, 640, None, 8, None) == 0
        for res_ld, total_ld, y_ld, q_ld, s_ld in ((0, 0, 320, 0, 0), (0, 0, 0, 384, 4), (320, 320, 328, 0, 0), (328, 320, 0, 384, 4), (320, 0, 336, 384, 4)):
            assert L.sige_token_rms(None, 1, 320, 320, None, res_ld, *rows, None, eps, None, total_ld, None, y_ld, None, q_ld, None, s_ld, None) == 0, (rows, y_ld, err(L))
            assert L.sige_token_rms(FAKE, 1, 320, 320, None, res_ld, *rows, None, eps, None, total_ld, None, y_ld, None, q_ld, None, s_ld, None) == 0


def test_binding_refuses_what_an_int_does_not_hold():
    """Sizes of 2^31 and more would reach the library as their lower 32 bits, and 2^32 + 5 rows be 5 (tensors without memory: nothing is read)."""
    big = 2 ** 32 + 5

    def tensor(*shape, dtype=torch.float16, strides=None):
        return torch.empty_strided(shape, strides or (shape[1], 1), dtype=dtype, device="meta")
    u8 = torch.uint8
    q, s = tensor(8, 128, dtype=u8), tensor(8, 4, dtype=u8)
    w, ws = tensor(64, 128, dtype=u8), tensor(64, 4, dtype=u8)
    x, y = tensor(8, 64), tensor(8, 32)
    count = torch.empty(1, dtype=torch.int32, device="meta")
    far = tensor(8, 64, strides=(2 ** 32 + 64, 1))
    qb, sb, xb, yb = tensor(big, 128, dtype=u8), tensor(big, 4, dtype=u8), tensor(big, 64), tensor(big, 32)
    wide, qw, sw = tensor(8, 2 ** 32 + 64), tensor(8, 2 ** 32 + 128, dtype=u8), tensor(8, 2 ** 25 + 4, dtype=u8)
    hw, hws = tensor(2 ** 33 + 64, 128, dtype=u8), tensor(2 ** 33 + 64, 4, dtype=u8)
    calls = [(api.sige_token_rms, (xb, 64), dict(y=xb, n_rows=big)), (api.sige_token_rms, (xb, 64), dict(y=xb, count=count, rows_per_count=16)),
             (api.sige_token_rms, (xb, 64), dict(y=xb, count=count, rows_per_count=16, max_rows=big)), (api.sige_token_rms, (x, 64), dict(y=far, n_rows=8)),
             (api.sige_token_rms, (x, 64), dict(y=x, residual=far, n_rows=8)), (api.sige_token_rms, (x, 64), dict(y=x, residual=x, total=far, n_rows=8)),
             (api.sige_token_rms, (wide, 2 ** 32 + 64), dict(y=wide, n_rows=8)), (api.sige_token_rms, (x, 64), dict(y=x, count=count, rows_per_count=2 ** 32 + 1)),
             (api.sige_rows8_store, (xb, qb, sb, 64), dict(n_rows=big)), (api.sige_rows8_store, (far, q, s, 64), dict(n_rows=8)),
             (api.sige_rows8_store, (wide, qw, sw, 2 ** 32 + 64), dict(n_rows=8)),
             (api.sige_rows8_load, (qb, sb, xb, 64), dict(n_rows=big)), (api.sige_rows8_load, (q, s, far, 64), dict(n_rows=8)),
             (api.sige_rows8_load, (tensor(8, 128, dtype=u8, strides=(2 ** 32 + 128, 1)), s, x, 64), dict(n_rows=8)),
             (api.sige_rows8_load, (q, tensor(8, 4, dtype=u8, strides=(2 ** 32 + 4, 1)), x, 64), dict(n_rows=8)),
             (api.sige_rows8_linear, (qb, sb, w, ws, yb, 64, 32), dict(n_rows=big)), (api.sige_rows8_linear, (q, s, w, ws, far, 64, 32), dict(n_rows=8)),
             (api.sige_rows8_linear, (q, s, w, ws, y, 64, 32), dict(n_rows=8, base=tensor(8, 32, strides=(2 ** 32 + 32, 1)))),
             (api.sige_rows8_linear, (q, s, hw, hws, tensor(8, 2 ** 32 + 32), 64, 2 ** 32 + 32), dict(n_rows=8)),
             (api.sige_rows8_linear_gated, (qb, sb, w, ws, qb, sb, 64, 32), dict(n_rows=big)),
             (api.sige_rows8_linear_gated, (q, s, hw, hws, qw, sw, 64, 2 ** 32 + 32), dict(n_rows=8)),
             (api.sige_rows8_linear_gated, (q, s, tensor(64, 128, dtype=u8, strides=(2 ** 32 + 128, 1)), ws, q, s, 64, 32), dict(n_rows=8))]
    for fn, a, kw in calls:
        with pytest.raises(api.SigeError) as e:
            fn(*a, **kw)
        assert e.value.code == 2 and "2^31" in str(e.value), (fn.__name__, e.value)
    with pytest.raises(api.SigeError, match="another device"):      # eight rows of a tensor of more than a call may have: nothing to refuse but the device
        api.sige_token_rms(xb, 64, y=xb, n_rows=8)

"""Token-wise layers on rows held in 8 bits, case by case: rows stored in 8 bits and read back, the root-mean-square norm with the
residual's addition and an output in 8 bits, the matrix product of two matrices in 8 bits, and the same product with a gated
activation behind it whose output is 8 bits again.

With ``own`` false, ``run`` computes them in their plain form with elementary torch operations in 32 bits; with ``own``
true it makes the calls a program makes of the library.  Everything is drawn on the GPU from the case's seed.

The format that the calls share with a program (include/sige.h): a matrix of rows x C is

codes    uint8 [rows][C rounded up to a multiple of 128]: e4m3, 0 behind C
scales   uint8 [rows][4 for every 512 channels begun]: byte s of a block of 128 channels is 2^(s - 127)

and what a case returns of it are the values it stands for.
"""
from __future__ import annotations

import math

import torch

own = False

DEV = "cuda"
DT = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
EPS = 1e-6
MOST = 448.0            # the largest number of e4m3
LEAST = -126            # the smallest exponent of a block


def listed():
    return [
        # the tokens of an edit (40 blocks of 4x4 of a 64x64 map) on their way into an 8-bit layer, and back: latency
        dict(name="rows_edit", kind="rows", dtype="bf16", rows=640, C=320),
        # a wide layer's tokens, or its weights when a model is opened: memory
        dict(name="rows_large", kind="rows", dtype="f16", rows=16384, C=5120),
        # one token between two layers
        dict(name="rms_one", kind="rms", dtype="bf16", rows=1, C=4096, residual=True, plain=False),
        # single precision, channels that do not fill their last block, both outputs, nothing added
        dict(name="rms_f32", kind="rms", dtype="f32", rows=1011, C=1288, residual=False, plain=True),
        # many tokens: memory
        dict(name="rms_large", kind="rms", dtype="bf16", rows=16384, C=2560, residual=True, plain=False),
        # one token through a wide layer: the weights' way from memory
        dict(name="linear_one", kind="linear", dtype="bf16", rows=1, cin=8192, cout=8192, bias=False, base=True),
        # one 4x4 block to queries, keys and values of a 1280-channel layer
        dict(name="linear_block", kind="linear", dtype="f16", rows=16, cin=1280, cout=3840, bias=True, base=False),
        # single precision, odd sizes, a residual
        dict(name="linear_f32", kind="linear", dtype="f32", rows=333, cin=1288, cout=648, bias=True, base=True),
        # many tokens of a wide layer: the matrix pipes
        dict(name="linear_large", kind="linear", dtype="bf16", rows=8192, cin=5120, cout=5120, bias=True, base=True),
        # one 4x4 block through the first feed-forward layer of a 1280-channel layer
        dict(name="gated_block", kind="gated", rows=16, cin=1280, cout=5120, act="gelu", bias=True),
        # a 15 % edit of a 64x64 map, 640 channels
        dict(name="gated_edit", kind="gated", rows=614, cin=640, cout=2560, act="gelu", bias=True),
        # the largest
        dict(name="gated_large", kind="gated", rows=4096, cin=2560, cout=10240, act="silu", bias=False),
    ]


def _log(rng, lo, hi):
    return min(hi, max(lo, round(math.exp(rng.uniform(math.log(lo), math.log(hi))))))


def draw(rng):
    kind = rng.choice(("rows", "rms", "linear", "linear", "gated", "gated"))
    dtype = rng.choice(("bf16", "f16", "f32"))
    if kind in ("rows", "rms"):
        C = 8 * _log(rng, 1, 1024)
        rows = _log(rng, 1, max(1, min(65536, (16384 * 2560 if kind == "rms" else 16384 * 5120) // (C * (2 if dtype == "f32" else 1)))))
        if kind == "rows":
            return dict(kind=kind, dtype=dtype, rows=rows, C=C)
        return dict(kind=kind, dtype=dtype, rows=rows, C=C, residual=rng.random() < 0.6, plain=rng.random() < 0.3)
    rows = _log(rng, 1, 8192)
    cin, cout = 8 * _log(rng, 2, 1024), 8 * _log(rng, 2, 1024)
    most = 8192 * 5120 * 5120 // (4 if kind == "linear" and dtype == "f32" else 2 if kind == "gated" else 1)
    rows = max(1, min(rows, most // (cin * cout)))
    if kind == "linear":
        return dict(kind=kind, dtype=dtype, rows=rows, cin=cin, cout=cout, bias=rng.random() < 0.5, base=rng.random() < 0.5)
    return dict(kind=kind, rows=rows, cin=cin, cout=cout, act=rng.choice(("gelu", "silu")), bias=rng.random() < 0.5)


# ---- inputs ------------------------------------------------------------------------------------------

def _exponents(g):
    """Of blocks [..., 128]: the smallest e with max|x| <= 448 * 2^e over the finite values."""
    a = g.abs()
    m, e = torch.frexp(torch.where(torch.isfinite(a), a, 0.0).amax(-1))     # max = m 2^e, m in [0.5, 1); 448 = 0.875 * 2^9
    return torch.where(m == 0, LEAST, torch.where(m > 0.875, e - 8, e - 9)).clamp(min=LEAST)


def _quantise(x):
    """[..., C] floats -> (e4m3 [..., blocks, 128], exponents [..., blocks]), to the nearest, ties to the even code."""
    g = torch.nn.functional.pad(x.float(), (0, -x.shape[-1] % 128)).unflatten(-1, (-1, 128))
    e = _exponents(g)
    return torch.ldexp(g, -e.unsqueeze(-1)).to(torch.float8_e4m3fn), e


def _matrix(x):
    """(codes, scales) of the rows of x in the library's format."""
    q, e = _quantise(x)
    scales = torch.zeros(x.shape[0], -(-x.shape[1] // 512) * 4, dtype=torch.uint8, device=DEV)
    scales[:, :e.shape[1]] = (e + 127).to(torch.uint8)
    return q.flatten(-2).view(torch.uint8), scales


def _values(codes, scales, C):
    """The numbers a matrix stands for."""
    blocks = codes.view(torch.float8_e4m3fn).float().unflatten(-1, (-1, 128))
    return torch.ldexp(blocks, scales[:, :blocks.shape[1]].int().unsqueeze(-1) - 127).flatten(-2)[:, :C]


def prepare(case, seed):
    torch.manual_seed(seed)
    torch.cuda.manual_seed(seed)
    s = dict(case)
    td = DT[case.get("dtype", "bf16")]
    randn = lambda *shape: torch.randn(*shape, device=DEV)  # noqa: E731
    if case["kind"] in ("rows", "rms"):
        # channels of unlike size, as activations have them
        size = torch.exp(0.7 * randn(case["C"]))
        s["x"] = (randn(case["rows"], case["C"]) * size).to(td)
        if case["kind"] == "rms":
            s["residual_"] = (randn(case["rows"], case["C"]) * size).to(td) if case["residual"] else None
            s["gamma"] = 1.0 + 0.2 * randn(case["C"])
        return s
    rows, cin, cout = case["rows"], case["cin"], case["cout"] * (2 if case["kind"] == "gated" else 1)
    s["x"], s["x_scales"] = _matrix(randn(rows, cin) * torch.exp(0.5 * randn(cin)))
    w = torch.empty(cout, s["x"].shape[1], dtype=torch.uint8, device=DEV)
    ws = torch.empty(cout, s["x_scales"].shape[1], dtype=torch.uint8, device=DEV)
    for i in range(0, cout, 4096):
        w[i:i + 4096], ws[i:i + 4096] = _matrix(randn(min(4096, cout - i), cin) / math.sqrt(cin))
    s["w"], s["w_scales"] = w, ws
    s["bias_"] = 0.1 * randn(cout) if case["bias"] else None
    if case["kind"] == "linear":
        s["base_"] = randn(rows, cout).to(td) if case["base"] else None
    return s


# ---- one pass ----------------------------------------------------------------------------------------

def run(s):
    return {"rows": _rows, "rms": _rms, "linear": _linear, "gated": _gated}[s["kind"]](s)


def _rows(s):
    x, n, C = s["x"], s["rows"], s["C"]
    if own:
        from paper_2211_02048_amd import api
        q, scales = api.rows8(n, C, x.device)
        y = torch.empty_like(x)
        api.sige_rows8_store(x, q, scales, C, n_rows=n)
        api.sige_rows8_load(q, scales, y, C, n_rows=n)
        return y
    q, e = _quantise(x)
    return torch.ldexp(q.float(), e.unsqueeze(-1)).flatten(-2)[:, :C].to(x.dtype)


def _rms(s):
    x, n, C, res = s["x"], s["rows"], s["C"], s["residual_"]
    if own:
        from paper_2211_02048_amd import api
        q, scales = api.rows8(n, C, x.device)
        total = None if res is None else torch.empty_like(x)
        y = torch.empty_like(x) if s["plain"] else None
        back = torch.empty(n, C, dtype=torch.bfloat16, device=x.device)
        api.sige_token_rms(x, C, s["gamma"], EPS, residual=res, total=total, y=y, q=q, scales=scales, n_rows=n)
        api.sige_rows8_load(q, scales, back, C, n_rows=n)
        return total, y, back
    h = x if res is None else (x.float() + res.float()).to(x.dtype)
    f = h.float()
    f = f * torch.rsqrt(f.square().mean(-1, keepdim=True) + EPS) * s["gamma"]
    q, e = _quantise(f)
    back = torch.ldexp(q.float(), e.unsqueeze(-1)).flatten(-2)[:, :C].to(torch.bfloat16)      # (4 bits of significand: exact)
    return None if res is None else h, f.to(x.dtype) if s["plain"] else None, back


def _product(s):
    """The product's plain form, fp32 [rows][output channels], with the bias."""
    y = _values(s["x"], s["x_scales"], s["cin"]) @ _values(s["w"], s["w_scales"], s["cin"]).t()
    return y if s["bias_"] is None else y + s["bias_"]


def _linear(s):
    n, cin, cout, td = s["rows"], s["cin"], s["cout"], DT[s["dtype"]]
    if own:
        from paper_2211_02048_amd import api
        y = torch.empty(n, cout, dtype=td, device=s["x"].device)
        api.sige_rows8_linear(s["x"], s["x_scales"], s["w"], s["w_scales"], y, cin, cout, bias=s["bias_"], base=s["base_"], n_rows=n)
        return y
    y = _product(s)
    return (y if s["base_"] is None else y + s["base_"].float()).to(td)


def _gated(s):
    n, cin, cout = s["rows"], s["cin"], s["cout"]
    if own:
        from paper_2211_02048_amd import api
        q, scales = api.rows8(n, cout, s["x"].device)
        back = torch.empty(n, cout, dtype=torch.bfloat16, device=s["x"].device)
        api.sige_rows8_linear_gated(s["x"], s["x_scales"], s["w"], s["w_scales"], q, scales, cin, cout,
                                    gate=api.GATE_GELU if s["act"] == "gelu" else api.GATE_SILU, bias=s["bias_"], n_rows=n)
        api.sige_rows8_load(q, scales, back, cout, n_rows=n)
        return back
    u, g = _product(s).chunk(2, -1)
    v = u * (0.5 * g * torch.special.erfc(-g * math.sqrt(0.5)) if s["act"] == "gelu" else g * torch.sigmoid(g))
    q, e = _quantise(v)
    return torch.ldexp(q.float(), e.unsqueeze(-1)).flatten(-2)[:, :cout].to(torch.bfloat16)


# ---- what a pass cannot do without -------------------------------------------------------------------

def work(case):
    size = 4 if case.get("dtype") == "f32" else 2
    held = lambda C: C + -(-C // 128)  # noqa: E731      a row's codes and scales
    if case["kind"] == "rows":
        return {"bytes": 2 * case["rows"] * (case["C"] * size + held(case["C"])), "flops": 2 * case["rows"] * case["C"]}
    if case["kind"] == "rms":
        n, C = case["rows"], case["C"]
        passes = 1 + 2 * case["residual"] + case["plain"]
        return {"bytes": n * (passes * C * size + 2 * held(C) + 2 * C) + 4 * C, "flops": 5 * n * C}
    n, cin, cout = case["rows"], case["cin"], case["cout"]
    if case["kind"] == "linear":
        return {"bytes": (n + cout) * held(cin) + n * cout * size * (1 + case["base"]) + 4 * cout * case["bias"], "flops": 2.0 * n * cin * cout}
    return {"bytes": (n + 2 * cout) * held(cin) + n * (2 * held(cout) + 2 * cout) + 8 * cout * case["bias"], "flops": 4.0 * n * cin * cout}


# ---- the definition in 64 bits -----------------------------------------------------------------------

def _nearest(x):
    """The values that the rows of x (64 bits) become in 8 bits: codes as a list of numbers, the nearest looked up."""
    codes = torch.arange(127, device=DEV)
    mag = torch.where(codes < 8, codes / 512.0, 2.0 ** (codes // 8 - 7) * (1 + codes % 8 / 8.0)).double()
    edges = (mag[1:] + mag[:-1]) / 2
    out = torch.empty_like(x)
    for c in range(0, x.shape[1], 128):
        b = x[:, c:c + 128]
        top = b.abs().amax(1, keepdim=True)
        e = torch.ceil(torch.log2(top / MOST))
        e = torch.where(MOST * torch.exp2(e) < top, e + 1, torch.where(MOST * torch.exp2(e - 1) >= top, e - 1, e)).clamp(min=LEAST)
        a = b.abs() / torch.exp2(e)
        low = torch.bucketize(a, edges)                         # (an edge itself: the code below it)
        low = torch.where((low < 126) & (a == edges[low.clamp(max=125)]) & (low % 2 == 1), low + 1, low)
        out[:, c:c + 128] = torch.sign(b) * mag[low] * torch.exp2(e)
    return out


def _double(codes, scales, C):
    k = torch.arange(C, device=DEV)
    c = codes[:, :C].int()
    e, m = c >> 3 & 15, c & 7
    v = torch.where(e == 0, m / 512.0, torch.exp2(e.double() - 7) * (1 + m / 8.0)).double()
    return torch.where(c > 127, -v, v) * torch.exp2(scales[:, k // 128].double() - 127)


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "rows":
        return _nearest(s["x"].double())
    if case["kind"] == "rms":
        h = s["x"].double()
        if s["residual_"] is not None:
            h = (h + s["residual_"].double()).to(s["x"].dtype).double()
        n = h / ((h * h).sum(1, keepdim=True) / case["C"] + EPS).sqrt() * s["gamma"].double()
        return h if case["residual"] else None, n if case["plain"] else None, _nearest(n)
    w = _double(s["w"], s["w_scales"], case["cin"])
    y = torch.cat([_double(s["x"][i:i + 2048], s["x_scales"][i:i + 2048], case["cin"]) @ w.t() for i in range(0, case["rows"], 2048)])
    if s["bias_"] is not None:
        y += s["bias_"].double()
    if case["kind"] == "linear":
        return y if s["base_"] is None else y + s["base_"].double()
    u, g = y[:, :case["cout"]], y[:, case["cout"]:]
    return _nearest(u * g * (torch.special.ndtr(g) if case["act"] == "gelu" else 1 / (1 + torch.exp(-g))))

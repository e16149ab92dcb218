"""Thin ctypes binding of libsige_hip.so: the same entry points as include/sige.h.

Argument marshalling only.  Tensors are torch CUDA tensors used purely as device
memory; every call enqueues on torch's current stream and returns at once.  There
is no fallback: if the library has not been built, or a call is refused, a
:class:`SigeError` is raised.
"""
from __future__ import annotations

import ctypes
import functools
import os
from dataclasses import dataclass

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libsige_hip.so")

SIGE_F32, SIGE_F16, SIGE_BF16 = 0, 1, 2
ACT_NONE, ACT_SILU, ACT_RELU, ACT_LEAKY_RELU = 0, 1, 2, 3
ROPE_ADJACENT, ROPE_HALVES = 0, 1
GATE_GELU, GATE_SILU = 0, 1
_DT = {torch.float32: SIGE_F32, torch.float16: SIGE_F16, torch.bfloat16: SIGE_BF16}
STATUS = {0: "SIGE_OK", 1: "SIGE_ERR_INVALID_ARG", 2: "SIGE_ERR_UNSUPPORTED", 3: "SIGE_ERR_CAPACITY",
          4: "SIGE_ERR_HIP"}

EXPORTS = ["sige_reduce_mask", "sige_reduce_mask_workspace_bytes", "sige_reduce_mask_lists", "sige_gather", "sige_gather_modulated", "sige_conv", "sige_conv_workspace_bytes", "sige_conv_geglu", "sige_conv_scatter", "sige_scatter", "sige_fused_conv", "sige_fused_conv_pair", "sige_sparse_attn", "sige_sparse_attn_blocks",
           "sige_sparse_attn_workspace_bytes", "sige_token_norm", "sige_gather_token_norm", "sige_geglu", "sige_packed_weight_bytes", "sige_pack_weight",
           "sige_gn_stats", "sige_gn_stats_act", "sige_last_error", "sige_version", "sige_set_knob", "sige_get_knob", "sige_conv_plan", "sige_reduce_mask_noalloc", "sige_mark_blocks",
           "sige_fused_conv_pair_marked", "sige_rope_pairs", "sige_token_rope", "sige_token_rope_blocks", "sige_cache4_bytes",
           "sige_cache4_store", "sige_cache4_store_blocks", "sige_cache4_load", "sige_cache4_attn", "sige_cache4_attn_blocks",
           "sige_cache4_attn_workspace_bytes", "sige_token_lora", "sige_rows8_store", "sige_rows8_load", "sige_token_rms",
           "sige_rows8_linear", "sige_rows8_linear_gated"]

# sige_knob of the header
KNOBS = {"CONV_CFG": 0, "CONV_KC": 1, "CONV_SPLIT": 2, "CONV_HALF": 3, "CONV_SPLIT_WGS": 4, "CONV_POINTWISE": 5,
         "CONV_POINTWISE_W4": 6, "CONV_PAIR_WGS": 7, "ATTN_WGS": 8, "DIFF_LOADS": 9, "DIFF_WGS": 10, "CONV_LDS_PAD": 12,
         "CONV_DIRECT": 11, "CONV_AHEAD": 13, "CACHE4_MANY": 14, "ROWS8_FORM": 15}


class SigeError(RuntimeError):
    def __init__(self, code: int, msg: str):
        super().__init__(f"{STATUS.get(code, code)}: {msg}")
        self.code = code


class Geom(ctypes.Structure):
    """Mirror of sige_geom."""
    _fields_ = [(n, ctypes.c_int32) for n in
                ("H_in", "W_in", "H_out", "W_out", "block_h", "block_w", "k", "stride", "pad")]

    @property
    def tile_h(self):
        return (self.block_h - 1) * self.stride + self.k

    @property
    def tile_w(self):
        return (self.block_w - 1) * self.stride + self.k

    @property
    def grid_blocks(self):
        return -(-self.H_out // self.block_h) * -(-self.W_out // self.block_w)


class BlockListDesc(ctypes.Structure):
    """Mirror of sige_block_list."""
    _fields_ = [("g", Geom), ("indices", ctypes.c_void_p), ("max_blocks", ctypes.c_int32),
                ("count", ctypes.c_void_p), ("workspace", ctypes.c_void_p), ("workspace_bytes", ctypes.c_size_t)]


class ConvPlanInfo(ctypes.Structure):
    """Mirror of sige_conv_plan_info."""
    _fields_ = [(n, ctypes.c_int32) for n in
                ("kernel", "shape", "patch_m", "patch_n", "k_steps_per_chunk", "ksplit", "workgroups", "threads",
                 "lds_bytes")]

    def __repr__(self):
        kind = "few-row 1x1" if self.kernel else "tiled"
        return (f"{kind} kernel, shape {self.shape} ({self.patch_m}x{self.patch_n}), {self.k_steps_per_chunk} K steps "
                f"per chunk, ksplit {self.ksplit}, {self.workgroups} workgroups of {self.threads}, {self.lds_bytes} B LDS")


def geom(H_in, W_in, block, k=3, stride=1, pad=None) -> Geom:
    pad = k // 2 if pad is None else pad
    bh, bw = (block, block) if isinstance(block, int) else block
    return Geom(H_in, W_in, (H_in + 2 * pad - k) // stride + 1, (W_in + 2 * pad - k) // stride + 1,
                bh, bw, k, stride, pad)


_lib = None


def lib() -> ctypes.CDLL:
    """Loads the HIP library; raises if it has not been built (no CPU fallback)."""
    global _lib
    if _recording is not None:
        return _recording
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise SigeError(-1, f"{LIB_PATH} is missing: run `python -m paper_2211_02048_amd.build` "
                                "(or __graft_entry__.build()) first")
        L = ctypes.CDLL(LIB_PATH)
        L.sige_last_error.restype = ctypes.c_char_p
        L.sige_packed_weight_bytes.restype = ctypes.c_size_t
        L.sige_sparse_attn_workspace_bytes.restype = ctypes.c_size_t
        vp, i32, f32, sz = ctypes.c_void_p, ctypes.c_int32, ctypes.c_float, ctypes.c_size_t
        gp = ctypes.POINTER(Geom)
        L.sige_reduce_mask.argtypes = [vp, vp, i32, i32, i32, i32, f32, vp, i32, i32, gp, vp, vp, i32, vp, vp, sz,
                                       vp]
        L.sige_reduce_mask_noalloc.argtypes = [vp, vp, i32, i32, i32, i32, f32, vp, i32, i32, gp, vp, vp, i32, vp, vp]
        L.sige_reduce_mask_lists.argtypes = [vp, vp, i32, i32, i32, i32, f32, vp, i32, i32,
                                             ctypes.POINTER(BlockListDesc), i32, vp, vp]
        L.sige_mark_blocks.argtypes = L.sige_reduce_mask_lists.argtypes
        L.sige_reduce_mask_workspace_bytes.restype = ctypes.c_size_t
        L.sige_reduce_mask_workspace_bytes.argtypes = [gp]
        L.sige_gather.argtypes = [vp, i32, i32, i32, i32, gp, vp, vp, i32, i32, vp, vp, i32, vp, vp]
        L.sige_gather_modulated.argtypes = [vp, i32, i32, i32, i32, gp, vp, vp, i32, i32, vp, vp, vp, i32, i32, vp, vp]
        L.sige_conv.argtypes = [vp, i32, gp, i32, i32, vp, vp, vp, i32, i32, vp, vp, sz, vp]
        L.sige_conv_geglu.argtypes = [vp, i32, gp, i32, i32, vp, vp, vp, i32, i32, vp, vp]
        L.sige_conv_scatter.argtypes = [vp, i32, gp, i32, i32, vp, vp, vp, vp, i32, i32, vp, vp, i32, vp, i32, vp, sz, vp]
        L.sige_conv_workspace_bytes.restype = ctypes.c_size_t
        L.sige_conv_workspace_bytes.argtypes = [i32, gp, i32, i32, i32]
        L.sige_fused_conv.argtypes = [vp, i32, i32, i32, i32, gp, vp, vp, i32, i32, vp, vp, i32, i32, vp, vp, vp, vp,
                                      i32, vp, i32, vp, vp, i32, vp, sz, vp]
        L.sige_fused_conv_pair.argtypes = [ctypes.POINTER(FusedConvCall), ctypes.POINTER(FusedConvCall), vp]
        L.sige_fused_conv_pair_marked.argtypes = [ctypes.POINTER(FusedConvCall), ctypes.POINTER(FusedConvCall),
                                                  ctypes.POINTER(BlockListDesc), vp]
        L.sige_scatter.argtypes = [vp, i32, gp, i32, vp, vp, i32, i32, vp, vp, i32, vp, i32, vp]
        L.sige_sparse_attn.argtypes = [vp, i32, vp, vp, i32, i32, i32, i32, i32, i32, f32, vp, i32, vp, sz, vp]
        L.sige_sparse_attn_workspace_bytes.argtypes = [i32, i32, i32, i32]
        L.sige_sparse_attn_blocks.argtypes = [vp, i32, gp, vp, i32, vp, vp, i32, i32, i32, i32, i32, f32, vp, i32, vp, sz, vp]
        L.sige_packed_weight_bytes.argtypes = [i32, i32, i32, i32]
        L.sige_pack_weight.argtypes = [vp, i32, i32, i32, i32, vp, vp]
        L.sige_token_norm.argtypes = [vp, i32, i32, i32, vp, i32, i32, i32, vp, vp, f32, vp, i32, vp]
        L.sige_gather_token_norm.argtypes = [vp, i32, i32, i32, gp, vp, vp, i32, i32, vp, vp, f32, vp, vp]
        L.sige_geglu.argtypes = [vp, i32, i32, i32, vp, i32, i32, i32, vp, i32, vp]
        L.sige_gn_stats.argtypes = [vp, i32, i32, i32, i32, i32, i32, vp, vp, f32, vp, vp, vp, vp, vp]
        L.sige_gn_stats_act.argtypes = [vp, i32, i32, i32, i32, i32, i32, vp, vp, f32, vp, vp, vp, vp, i32, vp, i32, vp]
        L.sige_conv_plan.argtypes = [i32, gp, i32, i32, i32, i32, i32, sz, ctypes.POINTER(ConvPlanInfo)]
        f64 = ctypes.c_double
        L.sige_rope_pairs.argtypes = [vp, i32, f64, vp]
        L.sige_token_rope.argtypes = [vp, i32, i32, i32, i32, vp, i32, i32, i32, vp, i32, i32, vp, i32, vp, i32, vp]
        L.sige_token_rope_blocks.argtypes = [vp, i32, i32, i32, i32, gp, vp, vp, i32, i32, vp, i32, i32, i32, f32, vp, i32, vp]
        L.sige_cache4_bytes.restype = L.sige_cache4_attn_workspace_bytes.restype = ctypes.c_size_t
        L.sige_cache4_bytes.argtypes = [i32, i32, i32]
        L.sige_cache4_store.argtypes = [vp, i32, vp, i32, i32, i32, i32, vp, i32, vp, i32, i32, i32, vp, i32, vp]
        L.sige_cache4_store_blocks.argtypes = [vp, i32, vp, i32, i32, i32, i32, gp, vp, vp, i32, i32, i32, vp, i32, vp]
        L.sige_cache4_load.argtypes = [vp, i32, i32, i32, i32, i32, i32, vp, i32, vp, i32, vp]
        L.sige_cache4_attn.argtypes = [vp, i32, vp, i32, i32, i32, i32, i32, i32, f32, vp, vp, i32, vp, sz, vp]
        L.sige_cache4_attn_blocks.argtypes = [vp, i32, gp, vp, i32, vp, i32, i32, i32, i32, i32, f32, vp, vp, i32, vp, sz, vp]
        L.sige_cache4_attn_workspace_bytes.argtypes = [i32, i32, i32, i32]
        L.sige_token_lora.argtypes = [vp, i32, i32, i32, vp, i32, i32, i32, vp, vp, i32, i32, vp, vp, vp, i32, i32, vp, i32, vp]
        L.sige_rows8_store.argtypes = [vp, i32, i32, i32, vp, i32, i32, i32, vp, i32, vp, i32, vp]
        L.sige_rows8_load.argtypes = [vp, i32, vp, i32, i32, vp, i32, i32, i32, vp, i32, i32, vp]
        L.sige_token_rms.argtypes = [vp, i32, i32, i32, vp, i32, vp, i32, i32, i32, vp, f32, vp, i32, vp, i32, vp, i32, vp, i32, vp]
        L.sige_rows8_linear.argtypes = [vp, i32, vp, i32, i32, vp, i32, i32, i32, vp, i32, vp, i32, i32, vp, vp, i32, vp, i32, i32, vp]
        L.sige_rows8_linear_gated.argtypes = [vp, i32, vp, i32, i32, vp, i32, i32, i32, vp, i32, vp, i32, i32, vp, i32, vp, i32, vp, i32, vp]
        L.sige_set_knob.argtypes = [i32, i32]
        L.sige_get_knob.argtypes = [i32]
        L.sige_get_knob.restype = i32
        _lib = L
    return _lib


# ---- prepared calls ---------------------------------------------------------------------------------
# A step that is a few kernels of a few microseconds each is bound by what the host does per launch.
# `record()` runs a piece of code once and keeps every library call it made together with its marshalled
# arguments; `CallList.run()` then repeats exactly those calls (same pointers, same sizes, same stream)
# without building the arguments again.  Marshalling only: each run still goes through the C entry
# points, which validate, plan and launch as always.
_QUERIES = ("sige_last_error", "sige_packed_weight_bytes", "sige_sparse_attn_workspace_bytes",
            "sige_reduce_mask_workspace_bytes", "sige_conv_workspace_bytes", "sige_conv_plan", "sige_set_knob",
            "sige_get_knob", "sige_rope_pairs", "sige_cache4_bytes", "sige_cache4_attn_workspace_bytes")


class CallList:
    """Library calls recorded by `record()`.  The tensors they name must outlive the list; the calls run
    on the stream that was current while they were recorded."""

    def __init__(self):
        self.calls = []

    def run(self):
        for fn, args in self.calls:
            rc = fn(*args)
            if rc != 0:
                _check(rc)

    def __len__(self):
        return len(self.calls)


class _RecordingLib:
    def __init__(self, real, calls):
        self._real, self._calls = real, calls

    def __getattr__(self, name):
        fn = getattr(self._real, name)
        if not name.startswith("sige_") or name in _QUERIES:
            return fn

        def call(*args):
            self._calls.append((fn, args))
            return fn(*args)
        return call


_recording = None


class record:
    """with api.record() as calls: ...   (the calls are made as usual and kept in `calls`)"""

    def __enter__(self):
        global _recording
        assert _recording is None, "api.record() does not nest"
        self.list = CallList()
        _recording = _RecordingLib(lib(), self.list.calls)
        return self.list

    def __exit__(self, *exc):
        global _recording
        _recording = None
        return False


def _ptr(t):
    return None if t is None else ctypes.c_void_p(t.data_ptr())


def _stream():
    return ctypes.c_void_p(torch.cuda.current_stream().cuda_stream)


def _check(rc: int):
    if rc != 0:
        raise SigeError(rc, lib().sige_last_error().decode())


def sige_reduce_mask_workspace_bytes(g: Geom) -> int:
    return int(lib().sige_reduce_mask_workspace_bytes(ctypes.byref(g)))


def sige_reduce_mask(g: Geom, indices, count, *, a_orig=None, a_edit=None, tau=0.0, mask_in=None,
                     mask_out=None, pool_log2=0, dilate=0, max_blocks=None, workspace=None):
    """Difference mask -> pooled, dilated mask -> ordered active-block list (device)."""
    if a_orig is not None:
        Hm, Wm, C = a_orig.shape
        dt = _DT[a_orig.dtype]
    else:
        Hm, Wm = mask_in.shape
        C, dt = 0, SIGE_F32
    mb = (indices.shape[0] if indices is not None else 0) if max_blocks is None else max_blocks
    _check(lib().sige_reduce_mask(_ptr(a_orig), _ptr(a_edit), dt, Hm, Wm, C, tau, _ptr(mask_in), pool_log2,
                                  dilate, ctypes.byref(g), _ptr(mask_out), _ptr(indices), mb, _ptr(count),
                                  _ptr(workspace), 0 if workspace is None else workspace.numel() *
                                  workspace.element_size(), _stream()))


NOALLOC_MAX_BLOCKS = 65536


def sige_reduce_mask_noalloc(g: Geom, indices, count, *, a_orig=None, a_edit=None, tau=0.0, mask_in=None,
                             mask_out=None, pool_log2=0, dilate=0, max_blocks=None):
    """sige_reduce_mask with the block flags in the library's built-in scratch: allocates nothing."""
    if a_orig is not None:
        Hm, Wm, C = a_orig.shape
        dt = _DT[a_orig.dtype]
    else:
        Hm, Wm = mask_in.shape
        C, dt = 0, SIGE_F32
    mb = indices.shape[0] if max_blocks is None else max_blocks
    _check(lib().sige_reduce_mask_noalloc(_ptr(a_orig), _ptr(a_edit), dt, Hm, Wm, C, tau, _ptr(mask_in), pool_log2,
                                          dilate, ctypes.byref(g), _ptr(mask_out), _ptr(indices), mb, _ptr(count),
                                          _stream()))


def sige_reduce_mask_lists(lists, *, a_orig=None, a_edit=None, tau=0.0, mask_in=None, mask_out=None,
                           pool_log2=0, dilate=0, mark_only=False):
    """One mask, several layer geometries: lists = [(g, indices, count, max_blocks, workspace), ...]."""
    if a_orig is not None:
        Hm, Wm, C = a_orig.shape
        dt = _DT[a_orig.dtype]
    else:
        Hm, Wm = mask_in.shape
        C, dt = 0, SIGE_F32
    arr = block_list_array(lists)
    fn = lib().sige_mark_blocks if mark_only else lib().sige_reduce_mask_lists
    _check(fn(_ptr(a_orig), _ptr(a_edit), dt, Hm, Wm, C, tau, _ptr(mask_in), pool_log2, dilate, arr, len(lists),
              _ptr(mask_out), _stream()))


def sige_mark_blocks(lists, **kw):
    """The first half of sige_reduce_mask_lists: mask and per-block flags, no lists (sige_fused_conv_pair_marked
    builds them)."""
    sige_reduce_mask_lists(lists, mark_only=True, **kw)


def block_list_array(lists):
    """[(g, indices, count, max_blocks, workspace), ...] as a host array of sige_block_list."""
    arr = (BlockListDesc * max(len(lists), 1))()
    for d, (g, indices, count, mb, ws) in zip(arr, lists):
        d.g = g
        d.indices, d.count = indices.data_ptr(), count.data_ptr()
        d.max_blocks = indices.shape[0] if mb is None else mb
        d.workspace = None if ws is None else ws.data_ptr()
        d.workspace_bytes = 0 if ws is None else ws.numel() * ws.element_size()
    arr._keep = lists
    return arr


def sige_gather(x, g: Geom, indices, count, tiles, *, n_blocks=-1, scale=None, shift=None, act=ACT_NONE,
                up=0, C=None, x_ld=None, max_blocks=None):
    """tiles[n] = act(scale * x[tile n] + shift), zero outside the image."""
    C = x.shape[-1] if C is None else C
    x_ld = x.stride(-2) if x_ld is None else x_ld
    mb = tiles.shape[0] if max_blocks is None else max_blocks
    _check(lib().sige_gather(_ptr(x), _DT[x.dtype], C, x_ld, up, ctypes.byref(g), _ptr(indices), _ptr(count),
                             mb, n_blocks, _ptr(scale), _ptr(shift), act, _ptr(tiles), _stream()))


def sige_gather_modulated(x, g: Geom, indices, count, tiles, mod, *, n_blocks=-1, scale=None, shift=None,
                          act=ACT_NONE, up=0, C=None, x_ld=None, mod_ld=None, max_blocks=None):
    """tiles[n] = act((scale * x + shift) * (1 + gamma) + beta) with per-pixel gamma | beta in mod [H, W, >=2C]."""
    C = x.shape[-1] if C is None else C
    x_ld = x.stride(-2) if x_ld is None else x_ld
    mod_ld = mod.stride(-2) if mod_ld is None else mod_ld
    mb = tiles.shape[0] if max_blocks is None else max_blocks
    _check(lib().sige_gather_modulated(_ptr(x), _DT[x.dtype], C, x_ld, up, ctypes.byref(g), _ptr(indices), _ptr(count),
                                       mb, n_blocks, _ptr(scale), _ptr(shift), _ptr(mod), mod_ld, act, _ptr(tiles),
                                       _stream()))


def _nbytes(t):
    return 0 if t is None else t.numel() * t.element_size()


def sige_conv_workspace_bytes(dtype, g: Geom, Cin, Cout, max_blocks) -> int:
    return int(lib().sige_conv_workspace_bytes(_DT[dtype], ctypes.byref(g), Cin, Cout, max_blocks))


def sige_conv_plan(dtype, g: Geom, Cin, Cout, n_blocks, *, staged_math=False, up=0, workspace_bytes=0) -> ConvPlanInfo:
    """Which kernel and launch shape a convolution call with these arguments would take (host only)."""
    info = ConvPlanInfo()
    _check(lib().sige_conv_plan(_DT[dtype], ctypes.byref(g), Cin, Cout, n_blocks, int(bool(staged_math)), up,
                                workspace_bytes, ctypes.byref(info)))
    return info


def sige_conv(tiles, g: Geom, Cin, Cout, packed_weight, bias, count, out_tiles, *, n_blocks=-1,
              max_blocks=None, workspace=None):
    """out_tiles[n] = valid conv of tiles[n] with the packed weight, plus bias."""
    mb = tiles.shape[0] if max_blocks is None else max_blocks
    _check(lib().sige_conv(_ptr(tiles), _DT[tiles.dtype], ctypes.byref(g), Cin, Cout, _ptr(packed_weight),
                           _ptr(bias), _ptr(count), mb, n_blocks, _ptr(out_tiles), _ptr(workspace),
                           _nbytes(workspace), _stream()))


def geglu_rows(n_out: int) -> torch.Tensor:
    """Row order sige_conv_geglu expects of a [2*n_out, ...] weight / bias whose first n_out rows are the
    values and whose last n_out rows are the gates: groups of 8 values followed by their 8 gates."""
    j = torch.arange(n_out).view(-1, 8)
    return torch.cat([j, j + n_out], dim=1).reshape(-1)


def sige_conv_geglu(tiles, g: Geom, Cin, Cout, packed_weight, bias, count, out_tiles, *, n_blocks=-1,
                    max_blocks=None):
    """out_tiles[n] = value * gelu(gate) of the 2*Cout-channel convolution of tiles[n] (weight rows in
    geglu_rows order)."""
    mb = tiles.shape[0] if max_blocks is None else max_blocks
    _check(lib().sige_conv_geglu(_ptr(tiles), _DT[tiles.dtype], ctypes.byref(g), Cin, Cout, _ptr(packed_weight),
                                 _ptr(bias), _ptr(count), mb, n_blocks, _ptr(out_tiles), _stream()))


def sige_conv_scatter(tiles, g: Geom, indices, count, Cin, Cout, packed_weight, bias, y, *, n_blocks=-1,
                      max_blocks=None, residual_tiles=None, residual=None, res_ld=None, y_ld=None, workspace=None):
    """conv on stacked tiles -> scatter in one call: y[block n] = conv(tiles[n]) (+ residuals), in place."""
    y_ld = y.stride(-2) if y_ld is None else y_ld
    if residual is not None and res_ld is None:
        res_ld = residual.stride(-2)
    mb = tiles.shape[0] if max_blocks is None else max_blocks
    _check(lib().sige_conv_scatter(_ptr(tiles), _DT[tiles.dtype], ctypes.byref(g), Cin, Cout, _ptr(packed_weight),
                                   _ptr(bias), _ptr(indices), _ptr(count), mb, n_blocks, _ptr(residual_tiles),
                                   _ptr(residual), res_ld or 0, _ptr(y), y_ld, _ptr(workspace), _nbytes(workspace),
                                   _stream()))


def sige_scatter(out_tiles, g: Geom, indices, count, y, *, n_blocks=-1, residual_tiles=None, residual=None,
                 Cout=None, y_ld=None, res_ld=None, max_blocks=None):
    """y[block n] = out_tiles[n] (+ residual_tiles[n]) (+ residual[block n]); y is updated in place."""
    Cout = out_tiles.shape[-1] if Cout is None else Cout
    y_ld = y.stride(-2) if y_ld is None else y_ld
    if residual is not None and res_ld is None:
        res_ld = residual.stride(-2)
    mb = out_tiles.shape[0] if max_blocks is None else max_blocks
    _check(lib().sige_scatter(_ptr(out_tiles), _DT[out_tiles.dtype], ctypes.byref(g), Cout, _ptr(indices),
                              _ptr(count), mb, n_blocks, _ptr(residual_tiles), _ptr(residual), res_ld or 0,
                              _ptr(y), y_ld, _stream()))


class ActOut(ctypes.Structure):
    """Mirror of sige_act_out."""
    _fields_ = [("y", ctypes.c_void_p), ("y_ld", ctypes.c_int32), ("scale", ctypes.c_void_p),
                ("shift", ctypes.c_void_p), ("act", ctypes.c_int32)]


class FusedConvCall(ctypes.Structure):
    """The arguments of one sige_fused_conv call (sige_fused_conv_call in the header)."""
    _fields_ = [("x", ctypes.c_void_p), ("dt", ctypes.c_int32), ("Cin", ctypes.c_int32), ("x_ld", ctypes.c_int32),
                ("up", ctypes.c_int32), ("g", ctypes.POINTER(Geom)), ("indices", ctypes.c_void_p),
                ("count", ctypes.c_void_p), ("max_blocks", ctypes.c_int32), ("n_blocks", ctypes.c_int32),
                ("scale", ctypes.c_void_p), ("shift", ctypes.c_void_p), ("act", ctypes.c_int32),
                ("Cout", ctypes.c_int32), ("packed_weight", ctypes.c_void_p), ("bias", ctypes.c_void_p),
                ("residual_tiles", ctypes.c_void_p), ("residual", ctypes.c_void_p), ("res_ld", ctypes.c_int32),
                ("y", ctypes.c_void_p), ("y_ld", ctypes.c_int32), ("out_tiles", ctypes.c_void_p),
                ("act_outs", ctypes.c_void_p), ("n_act_outs", ctypes.c_int32), ("workspace", ctypes.c_void_p),
                ("workspace_bytes", ctypes.c_size_t)]


def act_out_array(act_outs):
    """[(y, scale, shift, act), ...] (device tensors; y a [H, W, >=Cout] view) -> a ctypes array of sige_act_out."""
    arr = (ActOut * len(act_outs))()
    for a, (y, scale, shift, act) in zip(arr, act_outs):
        a.y, a.y_ld, a.scale, a.shift, a.act = _ptr(y), y.stride(-2), _ptr(scale), _ptr(shift), act
    return arr


def sige_fused_conv(x, g: Geom, indices, count, Cin, Cout, packed_weight, bias, *, y=None, out_tiles=None,
                    n_blocks=-1, max_blocks=None, scale=None, shift=None, act=ACT_NONE, up=0, x_ld=None,
                    residual_tiles=None, residual=None, res_ld=None, y_ld=None, workspace=None, act_outs=None):
    """gather -> conv -> scatter in one kernel; y is updated in place (or out_tiles receives the tiles).
    act_outs: [(y, scale, shift, act), ...] or a prepared act_out_array - activated copies of the output."""
    if act_outs is not None and not isinstance(act_outs, ctypes.Array):
        act_outs = act_out_array(act_outs)
    n_ao = 0 if act_outs is None else len(act_outs)
    x_ld = x.stride(-2) if x_ld is None else x_ld
    if y is not None and y_ld is None:
        y_ld = y.stride(-2)
    if residual is not None and res_ld is None:
        res_ld = residual.stride(-2)
    mb = indices.shape[0] if max_blocks is None else max_blocks
    _check(lib().sige_fused_conv(_ptr(x), _DT[x.dtype], Cin, x_ld, up, ctypes.byref(g), _ptr(indices), _ptr(count),
                                 mb, n_blocks, _ptr(scale), _ptr(shift), act, Cout, _ptr(packed_weight), _ptr(bias),
                                 _ptr(residual_tiles), _ptr(residual), res_ld or 0, _ptr(y), y_ld or 0,
                                 _ptr(out_tiles), act_outs if n_ao else None, n_ao, _ptr(workspace),
                                 _nbytes(workspace), _stream()))


def fused_conv_call(x, g: Geom, indices, count, Cin, Cout, packed_weight, bias, *, y=None, out_tiles=None,
                    n_blocks=-1, max_blocks=None, scale=None, shift=None, act=ACT_NONE, up=0, x_ld=None,
                    residual_tiles=None, residual=None, res_ld=None, y_ld=None, workspace=None, act_outs=None):
    """The arguments of sige_fused_conv as a FusedConvCall (keeps the tensors alive alongside)."""
    if act_outs is not None and not isinstance(act_outs, ctypes.Array):
        act_outs = act_out_array(act_outs)
    n_ao = 0 if act_outs is None else len(act_outs)
    if y is not None and y_ld is None:
        y_ld = y.stride(-2)
    if residual is not None and res_ld is None:
        res_ld = residual.stride(-2)
    p = lambda t: None if t is None else t.data_ptr()
    c = FusedConvCall(p(x), _DT[x.dtype], Cin, x.stride(-2) if x_ld is None else x_ld, up, ctypes.pointer(g),
                      p(indices), p(count), indices.shape[0] if max_blocks is None else max_blocks, n_blocks,
                      p(scale), p(shift), act, Cout, p(packed_weight), p(bias), p(residual_tiles), p(residual),
                      res_ld or 0, p(y), y_ld or 0, p(out_tiles),
                      ctypes.cast(act_outs, ctypes.c_void_p) if n_ao else None, n_ao, p(workspace),
                      _nbytes(workspace))
    c._keep = (x, g, indices, count, scale, shift, packed_weight, bias, residual_tiles, residual, y, out_tiles,
               act_outs, workspace)
    return c


def sige_fused_conv_pair(first: FusedConvCall, second: FusedConvCall):
    """Two independent fused calls; one launch when both take the few-block kernel shape."""
    _check(lib().sige_fused_conv_pair(ctypes.byref(first), ctypes.byref(second), _stream()))


def sige_fused_conv_pair_marked(first: FusedConvCall, second: FusedConvCall, marked):
    """sige_fused_conv_pair on lists that sige_mark_blocks left marked (marked: the two lists as for
    sige_reduce_mask_lists); the launch builds the ordered lists itself when it can."""
    arr = marked if isinstance(marked, ctypes.Array) else block_list_array(marked)
    _check(lib().sige_fused_conv_pair_marked(ctypes.byref(first), ctypes.byref(second), arr, _stream()))


def sige_token_norm(x, y, C, *, n_rows=-1, count=None, rows_per_count=0, max_rows=None, gamma=None, beta=None,
                    eps=1e-5, x_ld=None, y_ld=None):
    """y[r] = layer_norm(x[r]) * gamma + beta for the token rows of stacked tiles (x, y: [rows, >=C])."""
    x2, y2 = x.reshape(-1, x.shape[-1]), y.reshape(-1, y.shape[-1])
    mr = x2.shape[0] if max_rows is None else max_rows
    _check(lib().sige_token_norm(_ptr(x), _DT[x.dtype], C, x2.stride(0) if x_ld is None else x_ld, _ptr(count),
                                 rows_per_count, mr, n_rows, _ptr(gamma), _ptr(beta), eps, _ptr(y),
                                 y2.stride(0) if y_ld is None else y_ld, _stream()))


def sige_gather_token_norm(x, g: Geom, indices, count, tiles, C, *, n_blocks=-1, max_blocks=None, gamma=None,
                           beta=None, eps=1e-5, x_ld=None):
    """tiles[n] = layer_norm over the channels of every pixel of block n of x (gather and token norm in one)."""
    mb = tiles.shape[0] if max_blocks is None else max_blocks
    _check(lib().sige_gather_token_norm(_ptr(x), _DT[x.dtype], C, x.stride(-2) if x_ld is None else x_ld,
                                        ctypes.byref(g), _ptr(indices), _ptr(count), mb, n_blocks, _ptr(gamma),
                                        _ptr(beta), eps, _ptr(tiles), _stream()))


def sige_geglu(x, y, C, *, n_rows=-1, count=None, rows_per_count=0, max_rows=None, x_ld=None, y_ld=None):
    """y[r, c] = x[r, c] * gelu(x[r, C + c]) for the token rows of stacked tiles."""
    x2, y2 = x.reshape(-1, x.shape[-1]), y.reshape(-1, y.shape[-1])
    mr = x2.shape[0] if max_rows is None else max_rows
    _check(lib().sige_geglu(_ptr(x), _DT[x.dtype], C, x2.stride(0) if x_ld is None else x_ld, _ptr(count),
                            rows_per_count, mr, n_rows, _ptr(y), y2.stride(0) if y_ld is None else y_ld, _stream()))


def sige_sparse_attn_workspace_bytes(Nq, T, heads, d) -> int:
    return int(lib().sige_sparse_attn_workspace_bytes(Nq, T, heads, d))


def sige_sparse_attn(q, k, v, o, scale, *, Nq=None, workspace=None, heads=None, d=None, q_ld=None,
                     kv_ld=None, o_ld=None):
    """o[i, h] = softmax(scale * q[i, h] . k[:, h]) v[:, h] for the Nq edited query tokens."""
    heads = q.shape[1] if heads is None else heads
    d = q.shape[2] if d is None else d
    Nq = q.shape[0] if Nq is None else Nq
    T = k.shape[0]
    q_ld = q.stride(0) if q_ld is None else q_ld
    kv_ld = k.stride(0) if kv_ld is None else kv_ld
    o_ld = o.stride(0) if o_ld is None else o_ld
    wsb = 0 if workspace is None else workspace.numel() * workspace.element_size()
    _check(lib().sige_sparse_attn(_ptr(q), q_ld, _ptr(k), _ptr(v), kv_ld, _DT[q.dtype], Nq, T, heads, d,
                                  scale, _ptr(o), o_ld, _ptr(workspace), wsb, _stream()))


def sige_sparse_attn_blocks(q_full, g: Geom, indices, n_blocks, k, v, o, scale, *, heads, d, workspace=None,
                            q_ld=None, kv_ld=None, o_ld=None):
    """The same with the queries read from a full tensor by block list: query i is pixel
    i % (block_h*block_w) of block i / (block_h*block_w); o holds the stacked rows."""
    T = k.shape[0]
    q_ld = q_full.stride(-2) if q_ld is None else q_ld
    kv_ld = k.stride(0) if kv_ld is None else kv_ld
    o_ld = o.stride(0) if o_ld is None else o_ld
    wsb = 0 if workspace is None else workspace.numel() * workspace.element_size()
    _check(lib().sige_sparse_attn_blocks(_ptr(q_full), q_ld, ctypes.byref(g), _ptr(indices), n_blocks, _ptr(k),
                                         _ptr(v), kv_ld, _DT[q_full.dtype], T, heads, d, scale, _ptr(o), o_ld,
                                         _ptr(workspace), wsb, _stream()))


def sige_rope_pairs(axis_pairs, theta=10000.0, device="cuda") -> torch.Tensor:
    """The table of sige_token_rope, int32 [pairs][4] on `device`: the axes' pairs one after the other, axis_pairs[a] each,
    pair i of an axis with p pairs turning by theta^(-i / p) / (2 pi) turns per unit of position."""
    n = (ctypes.c_int32 * len(axis_pairs))(*axis_pairs)
    table = torch.zeros((max(sum(axis_pairs), 0), 4), dtype=torch.int32)
    _check(lib().sige_rope_pairs(n, len(axis_pairs), theta, _ptr(table)))
    return table.to(device)


# The wrappers below are called per layer and step, where the host's time is what a small call costs: pointers are passed as plain
# integers (the argtypes convert them), strides are read without making views.

def _stream_of(x, *tensors):
    """The current stream, on which the call will run; refuses tensors of another device than the current one (a CPU tensor's address
    is nothing a kernel may read)."""
    dev = x.get_device()
    for t in tensors:
        if t is not None and t.get_device() != dev:
            raise SigeError(1, f"tensors on {x.device} and on {t.device} in one call")
    if dev < 0 or dev != torch._C._cuda_getDevice():
        raise SigeError(1, f"a tensor on {x.device} in a call on another device")
    return torch._C._cuda_getCurrentRawStream(dev)


def _at(t):
    return None if t is None else t.data_ptr()


_I32 = torch.int32


def _like(x, *tensors):
    """The tensors a kernel takes for the type of x."""
    dtype = x.dtype
    for t in tensors:
        if t is not None and t.dtype is not dtype:
            raise SigeError(1, f"{t.dtype} beside {x.dtype} in one call")


def _table(what, t, dtype, n):
    """A table the kernels read entry by entry: at least n of them, one after the other."""
    if t.dtype is not dtype or t.numel() < n or not t.is_contiguous():
        raise SigeError(1, f"{what}: {n} entries of {dtype}, contiguous, not {tuple(t.shape)} of {t.dtype}")


def _holds(t, rows, width, ld=None):
    """Refuses a tensor that has not the rows a call touches: by its shape, or, where the call gives the rows' stride itself, by
    what its storage holds from its first element on."""
    if rows <= 0:
        return
    if ld is not None:
        room = t.untyped_storage().nbytes() // t.element_size() - t.storage_offset()
        if (rows - 1) * ld + width > room:
            raise SigeError(3, f"{rows} rows of {width} channels, {ld} apart, in a tensor with {room} elements behind its first")
    elif t.shape[-1] < width or t.numel() // t.shape[-1] < rows:
        raise SigeError(3, f"{rows} rows of {width} channels in a tensor of {tuple(t.shape)}")


def _lines(t, rows, width, ld=None):
    """Stride of the rows of t, [..., channels] with `rows` rows or more, of `width` channels or more, that follow each other at one
    distance; ld: the caller's own."""
    st = t.stride()
    if ld is not None:
        _holds(t, rows, width, ld)
    elif len(st) == 2 and st[1] == 1:
        ld = st[0]
        if t.shape[0] < rows or t.shape[1] < width:
            _holds(t, rows, width)
    else:
        sh = t.shape
        outer = [(n, s) for n, s in zip(sh[:-1], st[:-1]) if n != 1]       # (the stride of an axis of one is nobody's)
        if len(st) < 2 or st[-1] != 1 or any(s != outer[i + 1][0] * outer[i + 1][1] for i, (_, s) in enumerate(outer[:-1])):
            raise SigeError(1, f"rows of channels at one distance, not {tuple(sh)} with strides {st}")
        _holds(t, rows, width)
        ld = outer[-1][1] if outer else st[-2]
    return ld


def _block_list(indices, count, n_blocks, max_blocks=None):
    """The most blocks of a list that a call may read."""
    mb = indices.shape[0] if max_blocks is None else max_blocks
    if indices.dtype is not _I32 or indices.numel() < 2 * (mb if n_blocks < 0 else n_blocks) or not indices.is_contiguous():
        _table("indices", indices, _I32, 2 * (mb if n_blocks < 0 else n_blocks))
    if count is not None:
        _table("count", count, _I32, 1)
    return mb


def sige_token_rope(x, y, heads, d, pairs, positions, *, layout=ROPE_ADJACENT, n_rows=-1, count=None, rows_per_count=0,
                    max_rows=None, x_ld=None, y_ld=None):
    """Rotates the `heads` heads of every row by the row's positions (fp32 [rows, axes]); y may be x."""
    _like(x, y)
    mr = x.numel() // max(x.shape[-1], 1) if max_rows is None else max_rows
    rows = mr if n_rows < 0 else n_rows
    _table("pairs", pairs, _I32, 4 * pairs.shape[0])
    _table("positions", positions, torch.float32, rows * positions.shape[-1])
    if count is not None:
        _table("count", count, _I32, 1)
    x_ld, y_ld = _lines(x, rows, heads * d, x_ld), _lines(y, rows, heads * d, y_ld)
    stream = _stream_of(x, y, pairs, positions, count)
    rc = lib().sige_token_rope(x.data_ptr(), _DT[x.dtype], heads, d, x_ld, _at(count),
                               rows_per_count, mr, n_rows, pairs.data_ptr(), pairs.shape[0], layout, positions.data_ptr(),
                               positions.shape[-1], y.data_ptr(), y_ld, stream)
    if rc:
        _check(rc)


def sige_token_rope_blocks(x, y, heads, d, pairs, g: Geom, indices, count, *, n_axes=2, frame=0.0, layout=ROPE_ADJACENT,
                           n_blocks=-1, max_blocks=None, x_ld=None, y_ld=None):
    """The same with the positions (y, x) or (frame, y, x) of the listed blocks' pixels."""
    _like(x, y)
    _table("pairs", pairs, _I32, 4 * pairs.shape[0])
    mb = _block_list(indices, count, n_blocks, max_blocks)
    rows = (mb if n_blocks < 0 else n_blocks) * g.block_h * g.block_w
    x_ld, y_ld = _lines(x, rows, heads * d, x_ld), _lines(y, rows, heads * d, y_ld)
    stream = _stream_of(x, y, pairs, indices, count)
    rc = lib().sige_token_rope_blocks(x.data_ptr(), _DT[x.dtype], heads, d, x_ld, ctypes.byref(g),
                                      indices.data_ptr(), _at(count), mb, n_blocks, pairs.data_ptr(), pairs.shape[0], layout, n_axes,
                                      frame, y.data_ptr(), y_ld, stream)
    if rc:
        _check(rc)


@functools.lru_cache(maxsize=4096)
def sige_cache4_bytes(heads, d, capacity) -> int:
    """Bytes of a cache of `capacity` tokens' keys and values in 4 bits (0: not a head size the cache has)."""
    return int(lib().sige_cache4_bytes(heads, d, capacity))


def _rows_ld(t, rows, heads, d, ld=None):
    """Stride of the rows of t, [rows or more, heads * d or more] or [rows or more, heads, d]; ld: the caller's own."""
    if t is None:
        return 0
    if ld is not None:
        _holds(t, rows, heads * d, ld)
        return ld
    st, sh = t.stride(), t.shape
    if st[-1] != 1 or not (len(st) == 2 or len(st) == 3 and st[1] == d and sh[1:] == (heads, d)):
        raise SigeError(1, f"rows of {heads} heads of {d} channels, not {tuple(sh)} with strides {st}")
    if sh[0] < rows or len(st) == 2 and rows > 0 and sh[1] < heads * d:
        raise SigeError(3, f"{rows} rows of {heads} heads of {d} channels in a tensor of {tuple(sh)}")
    return st[0]


def _work_bytes(workspace):
    if workspace is not None and not workspace.is_contiguous():
        raise SigeError(1, "the workspace must be contiguous")
    return _nbytes(workspace)


def _check_cache(cache, heads, d, capacity):
    if not cache.is_contiguous():
        raise SigeError(1, "the cache must be contiguous")
    need = sige_cache4_bytes(heads, d, capacity)
    if _nbytes(cache) < need:
        raise SigeError(3, f"a cache of {capacity} tokens takes {need} bytes, the tensor has {_nbytes(cache)}")


def sige_cache4_store(k, v, cache, capacity, heads, d, *, slots=None, first=0, n_rows=-1, count=None, rows_per_count=0,
                      max_rows=None, k_ld=None, v_ld=None):
    """Rows of keys and values into the cache: row r to token slots[r], or to first + r."""
    _check_cache(cache, heads, d, capacity)
    _like(k, v)
    mr = k.shape[0] if max_rows is None else max_rows
    rows = mr if n_rows < 0 else n_rows
    if slots is not None:
        _table("slots", slots, _I32, rows)
    if count is not None:
        _table("count", count, _I32, 1)
    k_ld, v_ld = _rows_ld(k, rows, heads, d, k_ld), _rows_ld(v, rows, heads, d, v_ld)
    stream = _stream_of(k, v, cache, slots, count)
    rc = lib().sige_cache4_store(k.data_ptr(), k_ld, v.data_ptr(), v_ld, _DT[k.dtype], heads, d, _at(slots), first,
                                 _at(count), rows_per_count, mr, n_rows, cache.data_ptr(), capacity, stream)
    if rc:
        _check(rc)


def sige_cache4_store_blocks(k, v, cache, capacity, heads, d, g: Geom, indices, count, *, n_blocks=-1, max_blocks=None, first=0,
                             k_ld=None, v_ld=None):
    """The stacked tokens of the listed blocks into the cache: pixel (y, x) to token first + y * W + x."""
    _check_cache(cache, heads, d, capacity)
    _like(k, v)
    mb = _block_list(indices, count, n_blocks, max_blocks)
    rows = (mb if n_blocks < 0 else n_blocks) * g.block_h * g.block_w
    k_ld, v_ld = _rows_ld(k, rows, heads, d, k_ld), _rows_ld(v, rows, heads, d, v_ld)
    stream = _stream_of(k, v, cache, indices, count)
    rc = lib().sige_cache4_store_blocks(k.data_ptr(), k_ld, v.data_ptr(), v_ld, _DT[k.dtype], heads, d, ctypes.byref(g),
                                        indices.data_ptr(), _at(count), mb, n_blocks, first, cache.data_ptr(), capacity, stream)
    if rc:
        _check(rc)


def sige_cache4_load(cache, capacity, heads, d, k, v, *, first=0, n_tokens=None, k_ld=None, v_ld=None):
    """Tokens first, first + 1, ... of the cache as rows of k's and v's type (either may be None)."""
    _check_cache(cache, heads, d, capacity)
    t = k if k is not None else v
    if t is None:
        raise SigeError(1, "sige_cache4_load: k or v is required")
    _like(t, v)
    n = t.shape[0] if n_tokens is None else n_tokens
    k_ld, v_ld = _rows_ld(k, n, heads, d, k_ld), _rows_ld(v, n, heads, d, v_ld)
    stream = _stream_of(cache, k, v)
    rc = lib().sige_cache4_load(cache.data_ptr(), capacity, _DT[t.dtype], heads, d, first, n, _at(k), k_ld, _at(v), v_ld, stream)
    if rc:
        _check(rc)


def sige_cache4_attn_workspace_bytes(Nq, T, heads, d) -> int:
    return int(lib().sige_cache4_attn_workspace_bytes(Nq, T, heads, d))


def sige_cache4_attn(q, cache, capacity, o, scale, *, T, heads, d, Nq=None, ranges=None, workspace=None, q_ld=None, o_ld=None):
    """sige_sparse_attn on a cache in 4 bits; ranges (int32 [Nq, 2]): the tokens [begin, end) that each row sees."""
    _check_cache(cache, heads, d, capacity)
    _like(q, o)
    nq = q.shape[0] if Nq is None else Nq
    if ranges is not None:
        _table("ranges", ranges, _I32, 2 * nq)
    q_ld, o_ld, wsb = _rows_ld(q, nq, heads, d, q_ld), _rows_ld(o, nq, heads, d, o_ld), _work_bytes(workspace)
    stream = _stream_of(q, cache, o, ranges, workspace)
    rc = lib().sige_cache4_attn(q.data_ptr(), q_ld, cache.data_ptr(), capacity, _DT[q.dtype], nq, T, heads, d, scale, _at(ranges),
                                o.data_ptr(), o_ld, _at(workspace), wsb, stream)
    if rc:
        _check(rc)


def sige_cache4_attn_blocks(q_full, g: Geom, indices, n_blocks, cache, capacity, o, scale, *, T, heads, d, ranges=None,
                            workspace=None, q_ld=None, o_ld=None):
    """The same with the queries read from a full tensor by block list (sige_sparse_attn_blocks)."""
    _check_cache(cache, heads, d, capacity)
    _like(q_full, o)
    _block_list(indices, None, n_blocks)
    nq = n_blocks * g.block_h * g.block_w
    if ranges is not None:
        _table("ranges", ranges, _I32, 2 * nq)
    q_ld, o_ld = _lines(q_full, g.H_in * g.W_in if nq > 0 else 0, heads * d, q_ld), _rows_ld(o, nq, heads, d, o_ld)
    wsb = _work_bytes(workspace)
    stream = _stream_of(q_full, cache, o, indices, ranges, workspace)
    rc = lib().sige_cache4_attn_blocks(q_full.data_ptr(), q_ld, ctypes.byref(g), indices.data_ptr(), n_blocks, cache.data_ptr(),
                                       capacity, _DT[q_full.dtype], T, heads, d, scale, _at(ranges), o.data_ptr(), o_ld,
                                       _at(workspace), wsb, stream)
    if rc:
        _check(rc)


def sige_token_lora(x, y, Cin, Cout, down, up, ids, rows_per_id, *, alpha=None, base=None, n_rows=-1, count=None, max_rows=None,
                    x_ld=None, base_ld=None, y_ld=None):
    """y[r] = base[r] + alpha[i] * up[i] (down[i] x[r]) with i = ids[r // rows_per_id]; y may be base."""
    n, rank, c = down.shape
    if c != Cin or up.shape != (n, Cout, rank) or not (down.is_contiguous() and up.is_contiguous()):
        raise SigeError(1, "sige_token_lora: down is [adapters, rank, Cin] and up [adapters, Cout, rank], contiguous")
    _like(x, y, down, up, base)
    mr = x.numel() // max(x.shape[-1], 1) if max_rows is None else max_rows
    rows = mr if n_rows < 0 else n_rows
    _table("ids", ids, _I32, -(-rows // max(rows_per_id, 1)))
    if alpha is not None:
        _table("alpha", alpha, torch.float32, n)
    if count is not None:
        _table("count", count, _I32, 1)
    x_ld, y_ld = _lines(x, rows, Cin, x_ld), _lines(y, rows, Cout, y_ld)
    base_ld = 0 if base is None else _lines(base, rows, Cout, base_ld)
    stream = _stream_of(x, y, down, up, ids, alpha, base, count)
    rc = lib().sige_token_lora(x.data_ptr(), _DT[x.dtype], Cin, x_ld, _at(count), rows_per_id, mr, n_rows, down.data_ptr(), up.data_ptr(),
                               rank, n, _at(alpha), ids.data_ptr(), _at(base), base_ld, Cout, y.data_ptr(), y_ld, stream)
    if rc:
        _check(rc)


# ---- rows in 8 bits ------------------------------------------------------------------------------------

def rows8_lds(C):
    """Codes and scale bytes that a row of C channels takes."""
    return -(-C // 128) * 128, -(-C // 512) * 4


def rows8(rows, C, device="cuda"):
    """Room for `rows` rows of C channels in 8 bits: codes and scales."""
    return (torch.empty((rows, C + 127 & -128), dtype=_U8, device=device), torch.empty((rows, (C + 511 & -512) >> 7), dtype=_U8, device=device))


_U8 = torch.uint8


def _rows8(what, q, scales, rows, C):
    """Row strides of a matrix in 8 bits, [rows or more, codes] and [rows or more, scale bytes]."""
    ld, sld = C + 127 & -128, (C + 511 & -512) >> 7
    if q.dtype is not _U8 or scales.dtype is not _U8:
        raise SigeError(1, f"{what}: codes and scales are {_U8}, not {q.dtype} and {scales.dtype}")
    if q.dim() != 2 or scales.dim() != 2:
        raise SigeError(1, f"{what}: codes [rows, codes] and scales [rows, bytes], not {tuple(q.shape)} and {tuple(scales.shape)}")
    (a, b), (c, d) = q.stride(), scales.stride()
    if b != 1 or d != 1:
        raise SigeError(1, f"{what}: codes and scale bytes of a row side by side, not with strides {q.stride()} and {scales.stride()}")
    (n, wide), (m, swide) = q.shape, scales.shape
    if n < rows or m < rows or wide < ld or swide < sld:
        raise SigeError(3, f"{what}: {rows} rows of {C} channels take codes [{rows}, {ld}] and scales [{rows}, {sld}], not "
                           f"{tuple(q.shape)} and {tuple(scales.shape)}")
    # (the stride of an axis of one is nobody's)
    return a if n > 1 else max(ld, a), c if m > 1 else max(sld, c)


def _int32(who, *sizes):
    """Sizes that reach the library as 32-bit integers (of a larger one their lower 32 bits would)."""
    if max(sizes) > 0x7fffffff:
        raise SigeError(2, f"{who}: sizes and strides below 2^31, not {max(sizes)}")


def _row_count(x, n_rows, max_rows, count):
    """The most rows that a call may have, and those that it may touch."""
    if max_rows is None:
        sh = x.shape
        max_rows = sh[0] if len(sh) == 2 else x.numel() // max(sh[-1], 1)
        if n_rows >= 0 and max_rows > n_rows:
            max_rows = n_rows                                          # (room for more is nothing the call has to know)
    if count is not None:
        _table("count", count, _I32, 1)
    return max_rows, max_rows if n_rows < 0 else n_rows


def sige_rows8_store(x, q, scales, C, *, n_rows=-1, count=None, rows_per_count=0, max_rows=None, x_ld=None):
    """Rows of x to 8 bits: codes q and scales."""
    mr, rows = _row_count(x, n_rows, max_rows, count)
    x_ld = _lines(x, rows, C, x_ld)
    q_ld, s_ld = _rows8("q", q, scales, rows, C)
    _int32("sige_rows8_store", C, x_ld, rows_per_count, mr, n_rows, q_ld, s_ld)
    stream = _stream_of(x, q, scales, count)
    rc = lib().sige_rows8_store(x.data_ptr(), _DT[x.dtype], C, x_ld, _at(count), rows_per_count, mr, n_rows, q.data_ptr(), q_ld,
                                scales.data_ptr(), s_ld, stream)
    if rc:
        _check(rc)


def sige_rows8_load(q, scales, y, C, *, n_rows=-1, count=None, rows_per_count=0, max_rows=None, y_ld=None):
    """Rows in 8 bits back to rows of y's type."""
    mr, rows = _row_count(y, n_rows, max_rows, count)
    y_ld = _lines(y, rows, C, y_ld)
    q_ld, s_ld = _rows8("q", q, scales, rows, C)
    _int32("sige_rows8_load", C, y_ld, rows_per_count, mr, n_rows, q_ld, s_ld)
    stream = _stream_of(y, q, scales, count)
    rc = lib().sige_rows8_load(q.data_ptr(), q_ld, scales.data_ptr(), s_ld, C, _at(count), rows_per_count, mr, n_rows, y.data_ptr(),
                               _DT[y.dtype], y_ld, stream)
    if rc:
        _check(rc)


def sige_token_rms(x, C, gamma=None, eps=1e-6, *, residual=None, total=None, y=None, q=None, scales=None, n_rows=-1, count=None,
                   rows_per_count=0, max_rows=None, x_ld=None, res_ld=None, total_ld=None, y_ld=None):
    """h = x + residual (to total), its root-mean-square norm times gamma to y and, in 8 bits, to q and scales."""
    _like(x, residual, total, y)
    mr, rows = _row_count(x, n_rows, max_rows, count)
    if gamma is not None:
        _table("gamma", gamma, torch.float32, C)
    if (q is None) != (scales is None):
        raise SigeError(1, "sige_token_rms: codes and scales go together")
    x_ld = _lines(x, rows, C, x_ld)
    res_ld = 0 if residual is None else _lines(residual, rows, C, res_ld)
    total_ld = 0 if total is None else _lines(total, rows, C, total_ld)
    y_ld = 0 if y is None else _lines(y, rows, C, y_ld)
    q_ld, s_ld = (0, 0) if q is None else _rows8("q", q, scales, rows, C)
    _int32("sige_token_rms", C, x_ld, res_ld, total_ld, y_ld, rows_per_count, mr, n_rows, q_ld, s_ld)
    stream = _stream_of(x, residual, total, y, q, scales, gamma, count)
    rc = lib().sige_token_rms(x.data_ptr(), _DT[x.dtype], C, x_ld, _at(residual), res_ld, _at(count), rows_per_count, mr, n_rows, _at(gamma),
                              eps, _at(total), total_ld, _at(y), y_ld, _at(q), q_ld, _at(scales), s_ld, stream)
    if rc:
        _check(rc)


def sige_rows8_linear(x, x_scales, w, w_scales, y, Cin, Cout, *, bias=None, base=None, n_rows=-1, count=None, rows_per_count=0,
                      max_rows=None, base_ld=None, y_ld=None):
    """y = x w^T + bias + base with x [rows, Cin] and w [Cout, Cin] in 8 bits."""
    _like(y, base)
    mr, rows = _row_count(y, n_rows, max_rows, count)
    if bias is not None:
        _table("bias", bias, torch.float32, Cout)
    y_ld = _lines(y, rows, Cout, y_ld)
    base_ld = 0 if base is None else _lines(base, rows, Cout, base_ld)
    (q_ld, s_ld), (w_ld, ws_ld) = _rows8("x", x, x_scales, rows, Cin), _rows8("w", w, w_scales, Cout, Cin)
    _int32("sige_rows8_linear", Cin, Cout, y_ld, base_ld, rows_per_count, mr, n_rows, q_ld, s_ld, w_ld, ws_ld)
    stream = _stream_of(y, x, x_scales, w, w_scales, bias, base, count)
    rc = lib().sige_rows8_linear(x.data_ptr(), q_ld, x_scales.data_ptr(), s_ld, Cin, _at(count), rows_per_count, mr, n_rows, w.data_ptr(),
                                 w_ld, w_scales.data_ptr(), ws_ld, Cout, _at(bias), _at(base), base_ld, y.data_ptr(), _DT[y.dtype], y_ld,
                                 stream)
    if rc:
        _check(rc)


def sige_rows8_linear_gated(x, x_scales, w, w_scales, q, scales, Cin, Cout, *, gate=GATE_GELU, bias=None, n_rows=-1, count=None,
                            rows_per_count=0, max_rows=None):
    """The product with the values (rows 0 .. Cout - 1 of w) times the activated gates (rows Cout .. 2 Cout - 1), in 8 bits to q and scales."""
    mr, rows = _row_count(q, n_rows, max_rows, count)
    if bias is not None:
        _table("bias", bias, torch.float32, 2 * Cout)
    (x_ld, xs_ld), (w_ld, ws_ld) = _rows8("x", x, x_scales, rows, Cin), _rows8("w", w, w_scales, 2 * Cout, Cin)
    q_ld, s_ld = _rows8("q", q, scales, rows, Cout)
    _int32("sige_rows8_linear_gated", Cin, Cout, rows_per_count, mr, n_rows, x_ld, xs_ld, w_ld, ws_ld, q_ld, s_ld)
    stream = _stream_of(q, scales, x, x_scales, w, w_scales, bias, count)
    rc = lib().sige_rows8_linear_gated(x.data_ptr(), x_ld, x_scales.data_ptr(), xs_ld, Cin, _at(count), rows_per_count, mr, n_rows,
                                       w.data_ptr(), w_ld, w_scales.data_ptr(), ws_ld, Cout, _at(bias), gate, q.data_ptr(), q_ld,
                                       scales.data_ptr(), s_ld, stream)
    if rc:
        _check(rc)


def sige_packed_weight_bytes(dtype, Cout, Cin, k) -> int:
    return int(lib().sige_packed_weight_bytes(_DT[dtype], Cout, Cin, k))


def sige_pack_weight(w_oihw):
    """Returns the weight re-laid for sige_conv (a new device buffer owned by the caller)."""
    Cout, Cin, k, _ = w_oihw.shape
    nbytes = sige_packed_weight_bytes(w_oihw.dtype, Cout, Cin, k)
    if nbytes == 0:
        raise SigeError(2, f"sige_pack_weight: unsupported shape {tuple(w_oihw.shape)} for {w_oihw.dtype}")
    packed = torch.empty(nbytes // w_oihw.element_size(), dtype=w_oihw.dtype, device=w_oihw.device)
    w = w_oihw.contiguous()
    _check(lib().sige_pack_weight(_ptr(w), _DT[w.dtype], Cout, Cin, k, _ptr(packed), _stream()))
    return packed


def sige_gn_stats(x, groups, mean, var, *, gamma=None, beta=None, eps=1e-5, scale=None, shift=None,
                  C=None, x_ld=None):
    """Group mean / biased variance of a full tensor and the folded per-channel scale / shift."""
    H, W = x.shape[0], x.shape[1]
    C = x.shape[2] if C is None else C
    x_ld = x.stride(1) if x_ld is None else x_ld
    _check(lib().sige_gn_stats(_ptr(x), _DT[x.dtype], H, W, C, x_ld, groups, _ptr(gamma), _ptr(beta), eps,
                               _ptr(mean), _ptr(var), _ptr(scale), _ptr(shift), _stream()))


def sige_gn_stats_act(x, groups, mean, var, scale, shift, out, *, act=ACT_NONE, gamma=None, beta=None, eps=1e-5,
                      C=None, x_ld=None, out_ld=None):
    """sige_gn_stats and out = act(scale * x + shift) of the whole tensor."""
    H, W = x.shape[0], x.shape[1]
    C = x.shape[2] if C is None else C
    x_ld = x.stride(1) if x_ld is None else x_ld
    out_ld = out.stride(1) if out_ld is None else out_ld
    _check(lib().sige_gn_stats_act(_ptr(x), _DT[x.dtype], H, W, C, x_ld, groups, _ptr(gamma), _ptr(beta), eps,
                                   _ptr(mean), _ptr(var), _ptr(scale), _ptr(shift), act, _ptr(out), out_ld, _stream()))


def sige_version() -> int:
    return int(lib().sige_version())


def sige_set_knob(name: str, value: int) -> None:
    """Overrides one launch heuristic (value < 0: automatic again); see sige_knob in the header."""
    _check(lib().sige_set_knob(KNOBS[name], value))


def sige_get_knob(name: str) -> int:
    return int(lib().sige_get_knob(KNOBS[name]))


class knobs:
    """with api.knobs(CONV_CFG=3, CONV_KC=16): ... - overrides for the duration of the block."""

    def __init__(self, **kv):
        self.kv = kv

    def __enter__(self):
        self.prev = {k: sige_get_knob(k) for k in self.kv}
        for k, v in self.kv.items():
            sige_set_knob(k, -1 if v is None else int(v))
        return self

    def __exit__(self, *exc):
        for k, v in self.prev.items():
            sige_set_knob(k, v)
        return False

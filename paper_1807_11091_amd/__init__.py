"""Python binding of libstructadmm (gfx950): the StructADMM hot path.

Thin ctypes marshalling over the C ABI in ``include/structadmm.h``: every
step runs in the library's HIP kernels; torch is used only for device memory
(tensor allocation) and streams.  There is no fallback: if the library is
missing or a call fails, an exception is raised.

Entry points (same names as the C ABI):
  project(layers, ws=None, stream=None)
  project_workspace(layers)
  dual_update(layers, stream=None)
  sgd_step(items, stream=None)
  compact(Z, groups, ..., ws=None, stream=None) -> (Wc, row_idx, col_ch, col_tap, sizes)
  pack_nhwc(X, keep=None, Cx=None, stream=None)
  conv_fwd(X, Wc, col_ch, col_tap, sizes, C, D, stride, pad, Y=None, stream=None, ldy=None)
  conv_plan / conv_tiles(Xp, sizes, C, D, stride, pad) -> dict
  csr(Z, kept_idx, row_ptr=None, col=None, val=None, stream=None) -> (row_ptr, col, val)
  conv_sparse_workspace(Xp, shape, groups, stride, pad, nnz)
  conv_sparse_fwd(Xp, row_ptr, col, val, shape, groups, stride, pad, Y=None, ws=None, stream=None)
  layer_norm_fwd(X, gamma=None, beta=None, eps=1e-5, ...) -> (Y, mean, rstd)
  layer_norm_bwd(dY, X, mean, rstd, gamma=None, dR=None, ...) -> (dX, dgamma, dbeta)
  linear_fwd(X, W, bias=None, R=None, act=ACT_NONE, ...) -> Y
  linear_bwd(dY, X, W, Z=None, act=ACT_NONE, ...) -> (dX, dW, dbias)
  glu_fwd(X, Wg, Wu, bg=None, bu=None, act=ACT_SILU, ...) -> H
  glu_bwd(dH, X, Wg, Wu, G, U, act=ACT_SILU, ...) -> (dX, dWg, dWu, dbg, dbu)
  rms_norm_fwd(X, gamma=None, R=None, eps=1e-5, ...) -> (Y, S, rstd, Q)
  rms_norm_bwd(dY, S, rstd, gamma=None, dR=None, ...) -> (dX, dgamma)
  quantize8(X, block_rows=1, ...) -> (Q, QT)
  linear8_fwd(X, W, bias=None, R=None, act=ACT_NONE, ...) -> (Y, Q)
  glu8_fwd(X, Wg, Wu, bg=None, bu=None, act=ACT_SILU, ...) -> (H, Q)
  matrix8(rows, cols, block_rows=1, ...) -> an uninitialised Matrix8
  product8_plan(M, N, K, gated=False, ...) -> dict: the kernel of linear8_fwd / glu8_fwd
  compacted_matrix(Wc, sizes, group=0) -> the [M, K] matrix of a compacted layer
"""
from __future__ import annotations

import ctypes
import os
from dataclasses import dataclass
from typing import List, NamedTuple, Optional, Sequence

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libstructadmm.so")

FILTER, CHANNEL, SHAPE, ELEMENT = 0, 1, 2, 3
MAX_CONV_GROUPS = 16
MAX_STRUCT_GROUPS = 8192
COMPACT_WS_BYTES = 4096
ERRORS = {-1: "SA_E_ARG", -2: "SA_E_ALIGN", -3: "SA_E_WORKSPACE", -4: "SA_E_UNSUPPORTED", -5: "SA_E_HIP"}

_vp = ctypes.c_void_p


class ProjectDesc(ctypes.Structure):
    _fields_ = [("A", ctypes.c_int64), ("B", ctypes.c_int64), ("C", ctypes.c_int64), ("D", ctypes.c_int64),
                ("groups", ctypes.c_int32), ("kind", ctypes.c_int32), ("k", ctypes.c_int64),
                ("W", _vp), ("U", _vp), ("in_ch_mask", _vp), ("Z", _vp), ("mask", _vp),
                ("kept_idx", _vp), ("scores", _vp), ("rho", ctypes.c_float), ("G", _vp)]


class DualDesc(ctypes.Structure):
    _fields_ = [("n", ctypes.c_int64), ("W", _vp), ("Z", _vp), ("U", _vp), ("rho", ctypes.c_float),
                ("G", _vp), ("update_dual", ctypes.c_int32)]


class SgdDesc(ctypes.Structure):
    _fields_ = [("A", ctypes.c_int64), ("B", ctypes.c_int64), ("C", ctypes.c_int64), ("D", ctypes.c_int64),
                ("kind", ctypes.c_int32), ("mask", _vp), ("W", _vp), ("Gf", _vp), ("Z", _vp), ("U", _vp),
                ("rho", ctypes.c_float), ("lr", ctypes.c_float)]


class CompactDesc(ctypes.Structure):
    _fields_ = [("A", ctypes.c_int64), ("B", ctypes.c_int64), ("C", ctypes.c_int64), ("D", ctypes.c_int64),
                ("groups", ctypes.c_int32), ("Z", _vp), ("row_mask", _vp), ("col_mask", _vp),
                ("chan_mask", _vp), ("in_ch_mask", _vp), ("in_compacted", ctypes.c_int32),
                ("Wc", _vp), ("row_idx", _vp), ("col_ch", _vp), ("col_tap", _vp), ("ws", _vp)]


_G = MAX_CONV_GROUPS


class CompactSizes(ctypes.Structure):
    _fields_ = [("groups", ctypes.c_int32), ("M", ctypes.c_int32 * _G), ("K", ctypes.c_int32 * _G),
                ("ldk", ctypes.c_int32 * _G), ("wc_offset", ctypes.c_int64 * _G),
                ("row_offset", ctypes.c_int32 * _G), ("col_offset", ctypes.c_int32 * _G),
                ("run", ctypes.c_int32 * _G), ("run_base", ctypes.c_int32 * _G),
                ("ch_lo", ctypes.c_int32 * _G), ("ch_span", ctypes.c_int32 * _G),
                ("kpad", ctypes.c_int32 * _G)]

    def as_dict(self):
        g = self.groups
        return {k: list(getattr(self, k))[:g] for k in
                ("M", "K", "ldk", "wc_offset", "row_offset", "col_offset", "run", "run_base",
                 "ch_lo", "ch_span", "kpad")}


class ConvDesc(ctypes.Structure):
    _fields_ = [("N", ctypes.c_int32), ("H", ctypes.c_int32), ("W", ctypes.c_int32), ("Cx", ctypes.c_int32),
                ("C", ctypes.c_int32), ("D", ctypes.c_int32), ("stride", ctypes.c_int32), ("pad", ctypes.c_int32),
                ("sizes", ctypes.POINTER(CompactSizes)), ("X", _vp), ("Wc", _vp), ("col_ch", _vp),
                ("col_tap", _vp), ("Y", _vp), ("ws", _vp), ("ws_bytes", ctypes.c_size_t),
                ("ldy", ctypes.c_int32)]


class ConvPlanInfo(ctypes.Structure):
    _fields_ = [("groups", ctypes.c_int32), ("path", ctypes.c_int32 * _G), ("ksplit", ctypes.c_int32),
                ("space_to_depth", ctypes.c_int32), ("ig_tile", ctypes.c_int32 * 4),
                ("footprint_tile", ctypes.c_int32 * 3)]


class ConvTileInfo(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in (
        "direct_pixels", "direct_filters", "direct_fetchers", "direct_slices", "direct_one_tap",
        "footprint_pixels", "footprint_filters", "footprint_pixel_waves", "footprint_filter_waves")]


# kernel paths of structadmm_conv_plan
CONV_NONE, CONV_DIRECT, CONV_DIRECT_IG, CONV_FOOTPRINT, CONV_GATHER = 0, 1, 2, 3, 4


class CsrDesc(ctypes.Structure):
    _fields_ = [("A", ctypes.c_int64), ("B", ctypes.c_int64), ("C", ctypes.c_int64), ("D", ctypes.c_int64),
                ("nnz", ctypes.c_int64), ("Z", _vp), ("kept_idx", _vp), ("row_ptr", _vp), ("col", _vp),
                ("val", _vp)]


class SparseConvDesc(ctypes.Structure):
    _fields_ = [("N", ctypes.c_int32), ("H", ctypes.c_int32), ("W", ctypes.c_int32), ("Cx", ctypes.c_int32),
                ("A", ctypes.c_int32), ("B", ctypes.c_int32), ("C", ctypes.c_int32), ("D", ctypes.c_int32),
                ("groups", ctypes.c_int32), ("stride", ctypes.c_int32), ("pad", ctypes.c_int32),
                ("nnz", ctypes.c_int64), ("X", _vp), ("row_ptr", _vp), ("col", _vp), ("val", _vp),
                ("Y", _vp), ("ws", _vp), ("ws_bytes", ctypes.c_size_t), ("reuse_ws", ctypes.c_int32)]


# element types and activations of the feed-forward operators
BF16, F16, F32 = 0, 1, 2
ACT_NONE, ACT_RELU, ACT_SIGMOID, ACT_SILU, ACT_GELU, ACT_GELU_TANH = range(6)
ACTS = {"none": ACT_NONE, "relu": ACT_RELU, "sigmoid": ACT_SIGMOID, "silu": ACT_SILU, "gelu": ACT_GELU,
        "gelu_tanh": ACT_GELU_TANH}
MAX_LD = 1 << 21

_i32, _i64, _sz = ctypes.c_int32, ctypes.c_int64, ctypes.c_size_t


class LayerNormDesc(ctypes.Structure):
    _fields_ = [("rows", _i64), ("cols", _i64), ("type", _i32), ("eps", ctypes.c_float), ("X", _vp), ("ldx", _i64),
                ("gamma", _vp), ("beta", _vp), ("Y", _vp), ("ldy", _i64), ("mean", _vp), ("rstd", _vp)]


class LayerNormBwdDesc(ctypes.Structure):
    _fields_ = [("rows", _i64), ("cols", _i64), ("type", _i32), ("dY", _vp), ("lddy", _i64), ("X", _vp), ("ldx", _i64),
                ("mean", _vp), ("rstd", _vp), ("gamma", _vp), ("dR", _vp), ("lddr", _i64), ("dX", _vp),
                ("lddx", _i64), ("dgamma", _vp), ("dbeta", _vp), ("ws", _vp), ("ws_bytes", _sz)]


class LinearDesc(ctypes.Structure):
    _fields_ = [("M", _i64), ("N", _i64), ("K", _i64), ("type", _i32), ("out_type", _i32), ("act", _i32), ("X", _vp),
                ("ldx", _i64), ("W", _vp), ("ldw", _i64), ("bias", _vp), ("R", _vp), ("ldr", _i64), ("Y", _vp),
                ("ldy", _i64), ("Z", _vp), ("ldz", _i64), ("ws", _vp), ("ws_bytes", _sz)]


class LinearBwdDesc(ctypes.Structure):
    _fields_ = [("M", _i64), ("N", _i64), ("K", _i64), ("type", _i32), ("dw_type", _i32), ("act", _i32), ("dY", _vp),
                ("lddy", _i64), ("Z", _vp), ("ldz", _i64), ("X", _vp), ("ldx", _i64), ("W", _vp), ("ldw", _i64),
                ("dX", _vp), ("lddx", _i64), ("dW", _vp), ("lddw", _i64), ("dbias", _vp), ("ws", _vp),
                ("ws_bytes", _sz)]


class GluDesc(ctypes.Structure):
    _fields_ = [("M", _i64), ("N", _i64), ("K", _i64), ("type", _i32), ("act", _i32), ("X", _vp), ("ldx", _i64),
                ("Wg", _vp), ("Wu", _vp), ("ldw", _i64), ("bg", _vp), ("bu", _vp), ("H", _vp), ("ldh", _i64),
                ("G", _vp), ("U", _vp), ("ldgu", _i64), ("ws", _vp), ("ws_bytes", _sz)]


class GluBwdDesc(ctypes.Structure):
    _fields_ = [("M", _i64), ("N", _i64), ("K", _i64), ("type", _i32), ("dw_type", _i32), ("act", _i32), ("dH", _vp),
                ("lddh", _i64), ("G", _vp), ("U", _vp), ("ldgu", _i64), ("X", _vp), ("ldx", _i64), ("Wg", _vp),
                ("Wu", _vp), ("ldw", _i64), ("dX", _vp), ("lddx", _i64), ("dWg", _vp), ("dWu", _vp), ("lddw", _i64),
                ("dbg", _vp), ("dbu", _vp), ("ws", _vp), ("ws_bytes", _sz)]


BLOCK = 128  # columns (and rows, of a square block) that share a scale of an 8-bit matrix


class Matrix8Arg(ctypes.Structure):
    _fields_ = [("codes", _vp), ("ld", _i64), ("scales", _vp), ("scale_row", _i64), ("scale_col", _i64)]


class RmsNormDesc(ctypes.Structure):
    _fields_ = [("rows", _i64), ("cols", _i64), ("type", _i32), ("eps", ctypes.c_float), ("X", _vp), ("ldx", _i64),
                ("R", _vp), ("ldr", _i64), ("gamma", _vp), ("S", _vp), ("lds", _i64), ("Y", _vp), ("ldy", _i64),
                ("Q", Matrix8Arg), ("rstd", _vp)]


class RmsNormBwdDesc(ctypes.Structure):
    _fields_ = [("rows", _i64), ("cols", _i64), ("type", _i32), ("dY", _vp), ("lddy", _i64), ("S", _vp), ("lds", _i64),
                ("rstd", _vp), ("gamma", _vp), ("dR", _vp), ("lddr", _i64), ("dX", _vp), ("lddx", _i64),
                ("dgamma", _vp), ("ws", _vp), ("ws_bytes", _sz)]


class Quantize8Desc(ctypes.Structure):
    _fields_ = [("rows", _i64), ("cols", _i64), ("type", _i32), ("block_rows", _i32), ("X", _vp), ("ldx", _i64),
                ("Q", Matrix8Arg), ("QT", Matrix8Arg)]


class Linear8Desc(ctypes.Structure):
    _fields_ = [("M", _i64), ("N", _i64), ("K", _i64), ("type", _i32), ("out_type", _i32), ("act", _i32),
                ("X", Matrix8Arg), ("W", Matrix8Arg), ("bias", _vp), ("R", _vp), ("ldr", _i64), ("Y", _vp),
                ("ldy", _i64), ("Z", _vp), ("ldz", _i64), ("Q", Matrix8Arg), ("ws", _vp), ("ws_bytes", _sz),
                ("exact", _i32)]


class Glu8Desc(ctypes.Structure):
    _fields_ = [("M", _i64), ("N", _i64), ("K", _i64), ("type", _i32), ("act", _i32), ("X", Matrix8Arg),
                ("Wg", Matrix8Arg), ("Wu", Matrix8Arg), ("bg", _vp), ("bu", _vp), ("H", _vp), ("ldh", _i64),
                ("G", _vp), ("U", _vp), ("ldgu", _i64), ("Q", Matrix8Arg), ("ws", _vp), ("ws_bytes", _sz),
                ("exact", _i32)]


class Product8PlanInfo(ctypes.Structure):
    _fields_ = [(n, _i32) for n in ("rows", "tile_n", "tile_m", "exact", "split", "joined")]


class StructAdmmError(RuntimeError):
    pass


_lib = None


def lib():
    """Loads libstructadmm.so (raises if it has not been built)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise StructAdmmError(f"{LIB_PATH} is missing: build it with paper_1807_11091_amd/build.py")
        L = ctypes.CDLL(LIB_PATH)
        L.structadmm_project_workspace.argtypes = [ctypes.POINTER(ProjectDesc), ctypes.c_int]
        L.structadmm_project_workspace.restype = ctypes.c_size_t
        L.structadmm_project.argtypes = [ctypes.POINTER(ProjectDesc), ctypes.c_int, _vp, ctypes.c_size_t, _vp]
        L.structadmm_project.restype = ctypes.c_int
        L.structadmm_project_noalloc.argtypes = [ctypes.POINTER(ProjectDesc), ctypes.c_int, _vp]
        L.structadmm_project_noalloc.restype = ctypes.c_int
        L.structadmm_dual_update.argtypes = [ctypes.POINTER(DualDesc), ctypes.c_int, _vp]
        L.structadmm_dual_update.restype = ctypes.c_int
        L.structadmm_sgd_step.argtypes = [ctypes.POINTER(SgdDesc), ctypes.c_int, _vp]
        L.structadmm_sgd_step.restype = ctypes.c_int
        L.structadmm_compact.argtypes = [ctypes.POINTER(CompactDesc), ctypes.POINTER(CompactSizes), _vp]
        L.structadmm_compact.restype = ctypes.c_int
        L.structadmm_compact_many.argtypes = [ctypes.POINTER(CompactDesc), ctypes.c_int32,
                                              ctypes.POINTER(CompactSizes), _vp]
        L.structadmm_compact_many.restype = ctypes.c_int
        L.structadmm_pack_nhwc.argtypes = [_vp, ctypes.c_int32, ctypes.c_int32, ctypes.c_int32, ctypes.c_int32,
                                           _vp, ctypes.c_int32, _vp, _vp]
        L.structadmm_pack_nhwc.restype = ctypes.c_int
        L.structadmm_conv_fwd.argtypes = [ctypes.POINTER(ConvDesc), _vp]
        L.structadmm_conv_fwd.restype = ctypes.c_int
        L.structadmm_conv_plan.argtypes = [ctypes.POINTER(ConvDesc), ctypes.POINTER(ConvPlanInfo)]
        L.structadmm_conv_plan.restype = ctypes.c_int
        L.structadmm_conv_tiles.argtypes = [ctypes.POINTER(ConvDesc), ctypes.POINTER(ConvTileInfo)]
        L.structadmm_conv_tiles.restype = ctypes.c_int
        L.structadmm_conv_workspace.argtypes = [ctypes.POINTER(ConvDesc)]
        L.structadmm_conv_workspace.restype = ctypes.c_size_t
        L.structadmm_csr.argtypes = [ctypes.POINTER(CsrDesc), _vp]
        L.structadmm_csr.restype = ctypes.c_int
        L.structadmm_conv_sparse_workspace.argtypes = [ctypes.POINTER(SparseConvDesc)]
        L.structadmm_conv_sparse_workspace.restype = ctypes.c_size_t
        L.structadmm_conv_sparse_fwd.argtypes = [ctypes.POINTER(SparseConvDesc), _vp]
        L.structadmm_conv_sparse_fwd.restype = ctypes.c_int
        for name, cls in (("layer_norm_fwd", LayerNormDesc), ("layer_norm_bwd", LayerNormBwdDesc),
                          ("linear_fwd", LinearDesc), ("linear_bwd", LinearBwdDesc), ("glu_fwd", GluDesc),
                          ("glu_bwd", GluBwdDesc), ("rms_norm_fwd", RmsNormDesc), ("rms_norm_bwd", RmsNormBwdDesc),
                          ("quantize8", Quantize8Desc), ("linear8_fwd", Linear8Desc), ("glu8_fwd", Glu8Desc)):
            f = getattr(L, f"structadmm_{name}")
            f.argtypes = [ctypes.POINTER(cls), _vp]
            f.restype = ctypes.c_int
        for name, cls in (("linear8", Linear8Desc), ("glu8", Glu8Desc)):
            f = getattr(L, f"structadmm_{name}_plan")
            f.argtypes = [ctypes.POINTER(cls), ctypes.POINTER(Product8PlanInfo)]
            f.restype = ctypes.c_int
        for name, cls in (("layer_norm_bwd", LayerNormBwdDesc), ("linear", LinearDesc), ("linear_bwd", LinearBwdDesc),
                          ("glu", GluDesc), ("glu_bwd", GluBwdDesc), ("rms_norm_bwd", RmsNormBwdDesc),
                          ("linear8", Linear8Desc), ("glu8", Glu8Desc)):
            f = getattr(L, f"structadmm_{name}_workspace")
            f.argtypes = [ctypes.POINTER(cls)]
            f.restype = ctypes.c_size_t
        L.structadmm_last_error.argtypes = []
        L.structadmm_last_error.restype = ctypes.c_char_p
        L.structadmm_version.argtypes = []
        L.structadmm_version.restype = ctypes.c_char_p
        _lib = L
    return _lib


def _check(rc: int, what: str):
    if rc != 0:
        msg = lib().structadmm_last_error().decode(errors="replace")
        raise StructAdmmError(f"{what} failed: {ERRORS.get(rc, rc)} ({rc}): {msg}")


def _ptr(t) -> Optional[int]:
    return None if t is None else t.data_ptr()


_raw_stream = None


def _stream(stream) -> Optional[int]:
    """The handle of a stream (None: torch's current one)."""
    global _raw_stream
    if stream is None:
        import torch
        if _raw_stream is None:
            # the handle alone: torch.cuda.current_stream() takes 2.6 us to wrap it
            _raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (
                lambda device: torch.cuda.current_stream(device).cuda_stream)
        return _raw_stream(torch.cuda.current_device())
    return stream if isinstance(stream, int) else stream.cuda_stream


def _empty(stream, shape, dtype, device):
    """Uninitialised memory for a call on ``stream`` (a torch stream, a raw handle
    or None for the current one).  It comes from that stream's own pool: a block
    of the current stream's pool may still be in use by work that waits there and
    that ``stream`` does not wait for.  The current stream is marked as a user,
    so that a result which it reads may be dropped right after."""
    import torch
    if stream is None or isinstance(stream, int) and stream == _stream(None):
        return torch.empty(shape, dtype=dtype, device=device)
    if isinstance(stream, int):
        stream = torch.cuda.ExternalStream(stream, device=device)
    with torch.cuda.stream(stream):
        t = torch.empty(shape, dtype=dtype, device=device)
    t.record_stream(torch.cuda.current_stream(device))
    return t


@dataclass
class ProjectLayer:
    """One layer of a projection call: tensors are torch device tensors."""
    W: "object"
    U: "object"
    Z: "object"
    mask: "object"
    kept_idx: "object"
    kind: int
    k: int
    groups: int = 1
    in_ch_mask: "object" = None
    scores: "object" = None
    rho: float = 0.0
    G: "object" = None

    def desc(self) -> ProjectDesc:
        A, B, C, D = self.W.shape
        return ProjectDesc(A, B, C, D, self.groups, self.kind, self.k, _ptr(self.W), _ptr(self.U),
                           _ptr(self.in_ch_mask), _ptr(self.Z), _ptr(self.mask), _ptr(self.kept_idx),
                           _ptr(self.scores), self.rho, _ptr(self.G))


def _descs(layers: Sequence[ProjectLayer]):
    arr = (ProjectDesc * len(layers))()
    for i, l in enumerate(layers):
        arr[i] = l.desc()
    return arr


def project_workspace(layers: Sequence[ProjectLayer]) -> int:
    return int(lib().structadmm_project_workspace(_descs(layers), len(layers)))


def project(layers: Sequence[ProjectLayer], ws=None, stream=None, descs=None):
    """structadmm_project over the layers; ``ws`` is a uint8 device tensor."""
    d = descs if descs is not None else _descs(layers)
    nbytes = 0 if ws is None else ws.numel() * ws.element_size()
    _check(lib().structadmm_project(d, len(layers), _ptr(ws), nbytes, _stream(stream)), "structadmm_project")


# scratch the library holds per GPU for project_noalloc (bytes)
PROJECT_NOALLOC_BYTES = 16 << 20


def project_noalloc(layers: Sequence[ProjectLayer], stream=None, descs=None):
    """structadmm_project_noalloc: the projection with no workspace argument
    and no device allocation (the library's fixed per-GPU scratch)."""
    d = descs if descs is not None else _descs(layers)
    _check(lib().structadmm_project_noalloc(d, len(d), _stream(stream)), "structadmm_project_noalloc")


def dual_descs(items) -> "ctypes.Array":
    """items: iterable of (W, Z, U, rho, G, update_dual)."""
    items = list(items)
    arr = (DualDesc * len(items))()
    for i, (W, Z, U, rho, G, upd) in enumerate(items):
        arr[i] = DualDesc(W.numel(), _ptr(W), _ptr(Z), _ptr(U), rho, _ptr(G), 1 if upd else 0)
    return arr


def dual_update(items, stream=None, descs=None):
    d = descs if descs is not None else dual_descs(items)
    _check(lib().structadmm_dual_update(d, len(d), _stream(stream)), "structadmm_dual_update")


def sgd_descs(items) -> "ctypes.Array":
    """items: iterable of (W, Gf, Z, U, mask, kind, rho, lr); W is [A,B,C,D];
    Z, U and mask may be None."""
    items = list(items)
    arr = (SgdDesc * len(items))()
    for i, (W, Gf, Z, U, mask, kind, rho, lr) in enumerate(items):
        A, B, C, D = W.shape
        arr[i] = SgdDesc(A, B, C, D, kind, _ptr(mask), _ptr(W), _ptr(Gf), _ptr(Z), _ptr(U), rho, lr)
    return arr


def sgd_step(items, stream=None, descs=None):
    """structadmm_sgd_step: W <- keep ? W - lr * (Gf + rho((W - Z) + U)) : 0, in place."""
    d = descs if descs is not None else sgd_descs(items)
    _check(lib().structadmm_sgd_step(d, len(d), _stream(stream)), "structadmm_sgd_step")


def compact(Z, groups: int = 1, row_mask=None, col_mask=None, chan_mask=None, in_ch_mask=None,
            in_compacted: bool = False, ws=None, stream=None, out=None):
    """structadmm_compact; returns (Wc, row_idx, col_ch, col_tap, sizes)."""
    import torch
    A, B, C, D = Z.shape
    dev = Z.device
    K = B * C * D
    if out is None:
        Wc = _empty(stream, A * ((K + 63) // 64 * 64), torch.uint16, dev)
        row_idx = _empty(stream, A, torch.int32, dev)
        col_ch = _empty(stream, groups * K, torch.int32, dev)
        col_tap = _empty(stream, groups * K, torch.int32, dev)
    else:
        Wc, row_idx, col_ch, col_tap = out
    if ws is None:
        ws = _empty(stream, COMPACT_WS_BYTES, torch.uint8, dev)
    desc = CompactDesc(A, B, C, D, groups, _ptr(Z), _ptr(row_mask), _ptr(col_mask), _ptr(chan_mask),
                       _ptr(in_ch_mask), 1 if in_compacted else 0, _ptr(Wc), _ptr(row_idx), _ptr(col_ch),
                       _ptr(col_tap), _ptr(ws))
    sizes = CompactSizes()
    _check(lib().structadmm_compact(ctypes.byref(desc), ctypes.byref(sizes), _stream(stream)), "structadmm_compact")
    return Wc, row_idx, col_ch, col_tap, sizes


def compact_many(items, ws=None, stream=None):
    """structadmm_compact_many: one call (one wait of the host) for many
    compactions.  items: dicts of compact()'s arguments (Z, groups, row_mask,
    col_mask, chan_mask, in_ch_mask, in_compacted, out); ws: uint8 scratch of
    len(items) * COMPACT_WS_BYTES (allocated here when None).  Returns the
    list of (Wc, row_idx, col_ch, col_tap, sizes), one per item."""
    import torch
    n = len(items)
    if n == 0:
        return []
    dev = items[0]["Z"].device
    if ws is None:
        ws = _empty(stream, n * COMPACT_WS_BYTES, torch.uint8, dev)
    elif ws.numel() * ws.element_size() < n * COMPACT_WS_BYTES:
        raise StructAdmmError(f"compact_many: ws must hold {n} x {COMPACT_WS_BYTES} bytes")
    descs = (CompactDesc * n)()
    sizes = (CompactSizes * n)()
    outs = []
    for i, it in enumerate(items):
        Z = it["Z"]
        A, B, C, D = Z.shape
        groups = it.get("groups", 1)
        K = B * C * D
        if it.get("out") is None:
            o = (_empty(stream, A * ((K + 63) // 64 * 64), torch.uint16, dev),
                 _empty(stream, A, torch.int32, dev),
                 _empty(stream, groups * K, torch.int32, dev),
                 _empty(stream, groups * K, torch.int32, dev))
        else:
            o = tuple(it["out"])
        outs.append(o)
        descs[i] = CompactDesc(A, B, C, D, groups, _ptr(Z), _ptr(it.get("row_mask")), _ptr(it.get("col_mask")),
                               _ptr(it.get("chan_mask")), _ptr(it.get("in_ch_mask")),
                               1 if it.get("in_compacted") else 0, _ptr(o[0]), _ptr(o[1]), _ptr(o[2]), _ptr(o[3]),
                               ws.data_ptr() + i * COMPACT_WS_BYTES)
    _check(lib().structadmm_compact_many(descs, n, sizes, _stream(stream)), "structadmm_compact_many")
    return [outs[i] + (CompactSizes.from_buffer_copy(sizes[i]),) for i in range(n)]


def pack_nhwc(X, keep=None, Cx: Optional[int] = None, out=None, stream=None):
    """fp32 NCHW -> bf16 NHWC (uint16 bits) with an optional channel keep mask."""
    import torch
    N, Cin, H, W = X.shape
    if Cx is None:
        Cx = Cin if keep is None else int(keep.count_nonzero().item())
    Xp = out if out is not None else _empty(stream, (N, H, W, Cx), torch.uint16, X.device)
    _check(lib().structadmm_pack_nhwc(_ptr(X), N, Cin, H, W, _ptr(keep), Cx, _ptr(Xp), _stream(stream)),
           "structadmm_pack_nhwc")
    return Xp


def conv_out_shape(N, H, W, C, D, stride, pad, sizes: CompactSizes):
    P = (H + 2 * pad - C) // stride + 1
    Q = (W + 2 * pad - D) // stride + 1
    return (N, P, Q, int(sum(sizes.M[g] for g in range(sizes.groups))))


def conv_desc(Xp, Wc, col_ch, col_tap, sizes: CompactSizes, C, D, stride, pad, Y, ws=None, ldy=0) -> ConvDesc:
    N, H, W, Cx = Xp.shape
    nbytes = 0 if ws is None else ws.numel() * ws.element_size()
    return ConvDesc(N, H, W, Cx, C, D, stride, pad, ctypes.pointer(sizes), _ptr(Xp), _ptr(Wc),
                    _ptr(col_ch), _ptr(col_tap), _ptr(Y), _ptr(ws), nbytes, ldy)


def conv_workspace(Xp, sizes: CompactSizes, C: int, D: int, stride: int, pad: int) -> int:
    """Scratch bytes structadmm_conv_fwd needs for this input and compaction."""
    N, H, W, Cx = Xp.shape
    d = ConvDesc(N, H, W, Cx, C, D, stride, pad, ctypes.pointer(sizes), 16, 16, 16, 16, 16, None, 0)
    return int(lib().structadmm_conv_workspace(ctypes.byref(d)))


def conv_plan(Xp, sizes: CompactSizes, C: int, D: int, stride: int, pad: int) -> dict:
    """structadmm_conv_plan: the kernels structadmm_conv_fwd takes (host only)."""
    N, H, W, Cx = Xp.shape if not isinstance(Xp, tuple) else Xp
    d = ConvDesc(N, H, W, Cx, C, D, stride, pad, ctypes.pointer(sizes), 16, 16, 16, 16, 16, None, 0)
    info = ConvPlanInfo()
    _check(lib().structadmm_conv_plan(ctypes.byref(d), ctypes.byref(info)), "structadmm_conv_plan")
    g = info.groups
    return {"path": list(info.path)[:g], "ksplit": info.ksplit, "space_to_depth": info.space_to_depth,
            "ig_tile": tuple(info.ig_tile), "footprint_tile": tuple(info.footprint_tile)}


def conv_tiles(Xp, sizes: CompactSizes, C: int, D: int, stride: int, pad: int) -> dict:
    """structadmm_conv_tiles: the tile shapes of that plan (host only).
    "direct_tile": pixels, filters, fetching wavefronts (0: k_conv), slices in
    LDS, slices within one tap; "footprint_shape": pixels, filters, wavefronts
    over the pixels, over the filters.  Zeros for a path that no group takes."""
    N, H, W, Cx = Xp.shape if not isinstance(Xp, tuple) else Xp
    d = ConvDesc(N, H, W, Cx, C, D, stride, pad, ctypes.pointer(sizes), 16, 16, 16, 16, 16, None, 0)
    t = ConvTileInfo()
    _check(lib().structadmm_conv_tiles(ctypes.byref(d), ctypes.byref(t)), "structadmm_conv_tiles")
    return {"direct_tile": (t.direct_pixels, t.direct_filters, t.direct_fetchers, t.direct_slices, t.direct_one_tap),
            "footprint_shape": (t.footprint_pixels, t.footprint_filters, t.footprint_pixel_waves,
                                t.footprint_filter_waves)}


def conv_fwd(Xp, Wc, col_ch, col_tap, sizes: CompactSizes, C: int, D: int, stride: int, pad: int,
             Y=None, ws=None, stream=None, desc: Optional[ConvDesc] = None, ldy: Optional[int] = None):
    """structadmm_conv_fwd; Xp bf16 NHWC (uint16), returns Y bf16 NHWC (uint16).
    ``ws``: uint8 device scratch of conv_workspace() bytes (allocated here when None).
    ``ldy``: output row pitch in elements (>= the output channels Cy); by default
    the last dimension of a given 4-d Y, else Cy.  Y is then [N, P, Q, ldy] whose
    channels [Cy, ldy) are padding (left unchanged or set to +0)."""
    import torch
    if desc is None:
        N, H, W, Cx = Xp.shape
        shape = conv_out_shape(N, H, W, C, D, stride, pad, sizes)
        Cy = shape[-1]
        if ldy is None:
            ldy = Y.shape[-1] if (Y is not None and Y.dim() == 4) else Cy
        if ldy < Cy:
            raise StructAdmmError(f"conv_fwd: ldy={ldy} is below the {Cy} output channels")
        if Y is None:
            Y = _empty(stream, shape[:3] + (ldy,), torch.uint16, Xp.device)
        elif Y.numel() < shape[0] * shape[1] * shape[2] * ldy or Y.dtype != torch.uint16:
            raise StructAdmmError(f"conv_fwd: Y must be uint16 with room for {shape[:3]} rows of {ldy}")
        if ws is None:
            need = conv_workspace(Xp, sizes, C, D, stride, pad)
            ws = _empty(stream, need, torch.uint8, Xp.device) if need else None
        desc = conv_desc(Xp, Wc, col_ch, col_tap, sizes, C, D, stride, pad, Y, ws, 0 if ldy == Cy else ldy)
    _check(lib().structadmm_conv_fwd(ctypes.byref(desc), _stream(stream)), "structadmm_conv_fwd")
    return Y


def csr(Z, kept_idx, nnz: Optional[int] = None, row_ptr=None, col=None, val=None, stream=None):
    """structadmm_csr: CSR (row_ptr int32 [A+1], col int32 [nnz], val bf16 bits
    uint16 [nnz]) of an element-wise pruned layer from its projection's
    ascending kept indices."""
    import torch
    A, B, C, D = Z.shape
    nnz = int(kept_idx.numel()) if nnz is None else int(nnz)
    dev = Z.device
    if row_ptr is None:
        row_ptr = _empty(stream, A + 1, torch.int32, dev)
    if col is None:
        col = _empty(stream, max(nnz, 1), torch.int32, dev)
    if val is None:
        val = _empty(stream, max(nnz, 1), torch.uint16, dev)
    d = CsrDesc(A, B, C, D, nnz, _ptr(Z), _ptr(kept_idx) if nnz else None, _ptr(row_ptr),
                _ptr(col) if nnz else None, _ptr(val) if nnz else None)
    _check(lib().structadmm_csr(ctypes.byref(d), _stream(stream)), "structadmm_csr")
    for t in (row_ptr, col, val):  # given ones too stay until the stream has written them
        if stream is not None and not isinstance(stream, int):
            t.record_stream(stream)
    return row_ptr, col, val


def sparse_conv_desc(Xp, row_ptr, col, val, shape, groups, stride, pad, nnz, Y, ws=None,
                     reuse_ws: bool = False) -> SparseConvDesc:
    N, H, W, Cx = Xp.shape
    A, B, C, D = shape
    nbytes = 0 if ws is None else ws.numel() * ws.element_size()
    return SparseConvDesc(N, H, W, Cx, A, B, C, D, groups, stride, pad, nnz, _ptr(Xp), _ptr(row_ptr),
                          _ptr(col) if nnz else None, _ptr(val) if nnz else None, _ptr(Y), _ptr(ws), nbytes,
                          1 if reuse_ws else 0)


def conv_sparse_workspace(Xp, shape, groups: int, stride: int, pad: int, nnz: int) -> int:
    """Scratch bytes structadmm_conv_sparse_fwd needs."""
    d = sparse_conv_desc(Xp, None, None, None, shape, groups, stride, pad, nnz, None)
    return int(lib().structadmm_conv_sparse_workspace(ctypes.byref(d)))


def conv_sparse_fwd(Xp, row_ptr, col, val, shape, groups: int, stride: int, pad: int, nnz: int,
                    Y=None, ws=None, reuse_ws: bool = False, stream=None, desc: Optional[SparseConvDesc] = None):
    """structadmm_conv_sparse_fwd; Xp bf16 NHWC (uint16), returns Y bf16 NHWC
    [N, P, Q, A] (uint16).  reuse_ws: ws holds the padded entries an earlier
    call with the same CSR and geometry built."""
    import torch
    if desc is None:
        N, H, W, Cx = Xp.shape
        A, B, C, D = shape
        if Y is None:
            P = (H + 2 * pad - C) // stride + 1
            Q = (W + 2 * pad - D) // stride + 1
            Y = _empty(stream, (N, P, Q, A), torch.uint16, Xp.device)
        if ws is None:
            need = conv_sparse_workspace(Xp, shape, groups, stride, pad, nnz)
            ws = _empty(stream, max(need, 256), torch.uint8, Xp.device)
        desc = sparse_conv_desc(Xp, row_ptr, col, val, shape, groups, stride, pad, nnz, Y, ws, reuse_ws)
    _check(lib().structadmm_conv_sparse_fwd(ctypes.byref(desc), _stream(stream)), "structadmm_conv_sparse_fwd")
    return Y


# ------------------------------------------------------ feed-forward operators
_type_codes = {}


def _type_code(t, what: str) -> int:
    """sa_type of a tensor: bfloat16 (or its bits as uint16, as compact writes them), float16 or float32."""
    if not _type_codes:
        import torch
        _type_codes.update({torch.bfloat16: BF16, torch.uint16: BF16, torch.float16: F16, torch.float32: F32})
    code = _type_codes.get(t.dtype)
    if code is None:
        raise StructAdmmError(f"{what}: unsupported type {t.dtype}")
    return code


def _matrix(t, rows: int, cols: int, code: int, dev, what: str) -> int:
    """Checks a [rows, cols] matrix argument with unit column stride; its row pitch."""
    if t.shape != (rows, cols):
        raise StructAdmmError(f"{what} must be [{rows}, {cols}], got {tuple(t.shape)}")
    if t.device != dev:
        raise StructAdmmError(f"{what} is on {t.device}, not {dev}")
    if _type_code(t, what) != code:
        raise StructAdmmError(f"{what} has type {t.dtype}, not the operands'")
    ld, step = t.stride()
    if step != 1 and cols > 1 and rows > 0:
        raise StructAdmmError(f"{what} must have unit column stride")
    if rows <= 1:
        return max(ld, cols) if ld <= MAX_LD else cols  # a single row has no pitch
    return ld


def _vector(t, n: int, dev, what: str):
    """Checks an optional float32 vector of n entries; its pointer."""
    if t is None:
        return None
    if t.shape != (n,) or _type_codes.get(t.dtype) != F32 or t.device != dev or (n > 1 and t.stride(0) != 1):
        raise StructAdmmError(f"{what} must be float32 [{n}] on {dev}, contiguous")
    return t.data_ptr()


def _rows_of(X, what: str):
    if X.dim() != 2 or not X.is_cuda:
        raise StructAdmmError(f"{what} must be a matrix in GPU memory, got {tuple(X.shape)} on {X.device}")
    return X.shape


def _optional(t, rows, cols, code, dev, what):
    """(pointer, pitch) of a matrix that may be None."""
    return (None, cols) if t is None else (t.data_ptr(), _matrix(t, rows, cols, code, dev, what))


def _new(stream, like, rows: int, cols: int, dtype=None):
    import torch
    dtype = dtype or like.dtype
    return _empty(stream, (rows, cols), torch.bfloat16 if dtype == torch.uint16 else dtype, like.device)


def _run(desc, name: str, ws_fn, ws, like, stream):
    """Gives the descriptor its workspace and makes the call."""
    if ws_fn is not None:
        if ws is None:
            need = ws_fn(ctypes.byref(desc))
            if need:
                import torch
                ws = _empty(stream, need, torch.uint8, like.device)
        if ws is not None:
            if ws.device != like.device or not ws.is_contiguous():
                raise StructAdmmError(f"{name}: ws must be contiguous and on {like.device}, not {ws.device}")
            desc.ws, desc.ws_bytes = ws.data_ptr(), ws.numel() * ws.element_size()
    _check(getattr(lib(), name)(ctypes.byref(desc), _stream(stream)), name)


def compacted_matrix(Wc, sizes: CompactSizes, group: int = 0):
    """The compacted matrix of a conv group as a bfloat16 [M, K] view of Wc with
    row pitch ldk: the W of linear_fwd and the Wg / Wu of glu_fwd."""
    import torch
    if not 0 <= group < sizes.groups:
        raise StructAdmmError(f"compacted_matrix: group {group} outside [0, {sizes.groups})")
    M, K, ldk, at = sizes.M[group], sizes.K[group], sizes.ldk[group], sizes.wc_offset[group]
    return Wc.view(torch.bfloat16)[at:at + M * ldk].view(M, ldk)[:, :K]


def layer_norm_fwd(X, gamma=None, beta=None, eps: float = 1e-5, Y=None, mean=None, rstd=None, stats: bool = True,
                   stream=None):
    """structadmm_layer_norm_fwd over the rows of X [rows, cols] (bfloat16, float16
    or float32); returns (Y, mean, rstd).  mean and rstd, which the backward pass
    reads, are None with stats=False."""
    import torch
    rows, cols = _rows_of(X, "layer_norm_fwd: X")
    dev, code = X.device, _type_code(X, "layer_norm_fwd: X")
    ldx = _matrix(X, rows, cols, code, dev, "layer_norm_fwd: X")
    if Y is None:
        Y = _new(stream, X, rows, cols)
    if stats and mean is None:
        mean = _empty(stream, rows, torch.float32, dev)
    if stats and rstd is None:
        rstd = _empty(stream, rows, torch.float32, dev)
    d = LayerNormDesc(rows, cols, code, eps, X.data_ptr(), ldx, _vector(gamma, cols, dev, "layer_norm_fwd: gamma"),
                      _vector(beta, cols, dev, "layer_norm_fwd: beta"), Y.data_ptr(),
                      _matrix(Y, rows, cols, code, dev, "layer_norm_fwd: Y"),
                      _vector(mean, rows, dev, "layer_norm_fwd: mean"),
                      _vector(rstd, rows, dev, "layer_norm_fwd: rstd"))
    _run(d, "structadmm_layer_norm_fwd", None, None, X, stream)
    return Y, mean, rstd


def layer_norm_bwd(dY, X, mean, rstd, gamma=None, dR=None, dX=None, dgamma=None, dbeta=None, params: bool = True,
                   ws=None, stream=None):
    """structadmm_layer_norm_bwd; returns (dX, dgamma, dbeta).  dR: the gradient
    that reaches X past the norm, added to dX.  dgamma and dbeta are None with
    params=False (unless given)."""
    import torch
    rows, cols = _rows_of(X, "layer_norm_bwd: X")
    dev, code, w = X.device, _type_code(X, "layer_norm_bwd: X"), "layer_norm_bwd: "
    if mean is None or rstd is None:
        raise StructAdmmError(w + "mean and rstd of the forward pass are required")
    if dX is None:
        dX = _new(stream, X, rows, cols)
    if params and dgamma is None:
        dgamma = _empty(stream, cols, torch.float32, dev)
    if params and dbeta is None:
        dbeta = _empty(stream, cols, torch.float32, dev)
    r, ldr = _optional(dR, rows, cols, code, dev, w + "dR")
    d = LayerNormBwdDesc(rows, cols, code, dY.data_ptr(), _matrix(dY, rows, cols, code, dev, w + "dY"), X.data_ptr(),
                         _matrix(X, rows, cols, code, dev, w + "X"), _vector(mean, rows, dev, w + "mean"),
                         _vector(rstd, rows, dev, w + "rstd"), _vector(gamma, cols, dev, w + "gamma"), r, ldr,
                         dX.data_ptr(), _matrix(dX, rows, cols, code, dev, w + "dX"),
                         _vector(dgamma, cols, dev, w + "dgamma"), _vector(dbeta, cols, dev, w + "dbeta"), None, 0)
    _run(d, "structadmm_layer_norm_bwd", lib().structadmm_layer_norm_bwd_workspace, ws, X, stream)
    return dX, dgamma, dbeta


def linear_fwd(X, W, bias=None, R=None, act: int = ACT_NONE, Y=None, Z=None, out_dtype=None, ws=None, stream=None):
    """structadmm_linear_fwd: Y = act(X W^T + bias) + R for X [M, K] and W [N, K]
    (bfloat16 or float16); returns Y [M, N] (the operands' type, or float32 with
    out_dtype=torch.float32 or a float32 Y; R has Y's type).  Z: receives the
    pre-activations, which linear_bwd reads."""
    M, K = _rows_of(X, "linear_fwd: X")
    N, _ = _rows_of(W, "linear_fwd: W")
    dev, code, w = X.device, _type_code(X, "linear_fwd: X"), "linear_fwd: "
    if Y is None:
        Y = _new(stream, X, M, N, out_dtype)
    out = _type_code(Y, w + "Y")
    r, ldr = _optional(R, M, N, out, dev, w + "R")
    z, ldz = _optional(Z, M, N, code, dev, w + "Z")
    d = LinearDesc(M, N, K, code, out, act, X.data_ptr(), _matrix(X, M, K, code, dev, w + "X"), W.data_ptr(),
                   _matrix(W, N, K, code, dev, w + "W"), _vector(bias, N, dev, w + "bias"), r, ldr, Y.data_ptr(),
                   _matrix(Y, M, N, out, dev, w + "Y"), z, ldz, None, 0)
    _run(d, "structadmm_linear_fwd", lib().structadmm_linear_workspace, ws, X, stream)
    return Y


def linear_bwd(dY, X, W, Z=None, act: int = ACT_NONE, dX=None, dW=None, dbias=None, grads: str = "xw", dw_dtype=None,
               ws=None, stream=None):
    """structadmm_linear_bwd; returns (dX, dW, dbias).  grads names the gradients to
    make besides the buffers given: "x", "w" and "b" (the others are None).  dW is
    float32 (the Gf of sgd_step) unless dw_dtype or a dW buffer says otherwise.
    Z: the pre-activations (not needed for ACT_NONE)."""
    import torch
    M, K = _rows_of(X, "linear_bwd: X")
    N, _ = _rows_of(W, "linear_bwd: W")
    dev, code, w = X.device, _type_code(X, "linear_bwd: X"), "linear_bwd: "
    if dX is None and "x" in grads:
        dX = _new(stream, X, M, K)
    if dW is None and "w" in grads:
        dW = _new(stream, X, N, K, dw_dtype or torch.float32)
    if dbias is None and "b" in grads:
        dbias = _empty(stream, N, torch.float32, dev)
    wcode = code if dW is None else _type_code(dW, w + "dW")
    z, ldz = _optional(Z, M, N, code, dev, w + "Z")
    dx, lddx = _optional(dX, M, K, code, dev, w + "dX")
    dw, lddw = _optional(dW, N, K, wcode, dev, w + "dW")
    d = LinearBwdDesc(M, N, K, code, wcode, act, dY.data_ptr(), _matrix(dY, M, N, code, dev, w + "dY"), z, ldz,
                      X.data_ptr(), _matrix(X, M, K, code, dev, w + "X"), W.data_ptr(),
                      _matrix(W, N, K, code, dev, w + "W"), dx, lddx, dw, lddw, _vector(dbias, N, dev, w + "dbias"),
                      None, 0)
    _run(d, "structadmm_linear_bwd", lib().structadmm_linear_bwd_workspace, ws, X, stream)
    return dX, dW, dbias


def _pair(A, B, rows, cols, code, dev, what):
    """The one pitch of two matrices."""
    a, b = _matrix(A, rows, cols, code, dev, what[0]), _matrix(B, rows, cols, code, dev, what[1])
    if a != b and rows > 1:
        raise StructAdmmError(f"{what[0]} and {what[1]} must have the same row pitch")
    return a


def glu_fwd(X, Wg, Wu, bg=None, bu=None, act: int = ACT_SILU, H=None, G=None, U=None, ws=None, stream=None):
    """structadmm_glu_fwd: H = act(X Wg^T + bg) * (X Wu^T + bu) for X [M, K], Wg and
    Wu [N, K] of one row pitch (bfloat16 or float16); returns H [M, N].  G and U
    (both or neither) receive the two projections, which glu_bwd reads."""
    M, K = _rows_of(X, "glu_fwd: X")
    N, _ = _rows_of(Wg, "glu_fwd: Wg")
    dev, code, w = X.device, _type_code(X, "glu_fwd: X"), "glu_fwd: "
    if (G is None) != (U is None):
        raise StructAdmmError(w + "give both G and U or neither")
    if H is None:
        H = _new(stream, X, M, N)
    ldgu = N if G is None else _pair(G, U, M, N, code, dev, (w + "G", w + "U"))
    d = GluDesc(M, N, K, code, act, X.data_ptr(), _matrix(X, M, K, code, dev, w + "X"), Wg.data_ptr(), Wu.data_ptr(),
                _pair(Wg, Wu, N, K, code, dev, (w + "Wg", w + "Wu")), _vector(bg, N, dev, w + "bg"),
                _vector(bu, N, dev, w + "bu"), H.data_ptr(), _matrix(H, M, N, code, dev, w + "H"), _ptr(G), _ptr(U),
                ldgu, None, 0)
    _run(d, "structadmm_glu_fwd", lib().structadmm_glu_workspace, ws, X, stream)
    return H


def glu_bwd(dH, X, Wg, Wu, G, U, act: int = ACT_SILU, dX=None, dWg=None, dWu=None, dbg=None, dbu=None,
            grads: str = "xw", dw_dtype=None, ws=None, stream=None):
    """structadmm_glu_bwd; returns (dX, dWg, dWu, dbg, dbu).  grads names the
    gradients to make besides the buffers given: "x", "w" (dWg and dWu) and "b"
    (dbg and dbu).  dWg and dWu are float32 views of one [N, 2K] matrix, neuron by
    neuron, unless dw_dtype or buffers say otherwise."""
    import torch
    M, K = _rows_of(X, "glu_bwd: X")
    N, _ = _rows_of(Wg, "glu_bwd: Wg")
    dev, code, w = X.device, _type_code(X, "glu_bwd: X"), "glu_bwd: "
    if (dWg is None) != (dWu is None):
        raise StructAdmmError(w + "give both dWg and dWu or neither")
    if dX is None and "x" in grads:
        dX = _new(stream, X, M, K)
    if dWg is None and "w" in grads:
        dW = _new(stream, X, N, 2 * K, dw_dtype or torch.float32)
        dWg, dWu = dW[:, :K], dW[:, K:]
    if dbg is None and "b" in grads:
        dbg = _empty(stream, N, torch.float32, dev)
    if dbu is None and "b" in grads:
        dbu = _empty(stream, N, torch.float32, dev)
    wcode = code if dWg is None else _type_code(dWg, w + "dWg")
    dx, lddx = _optional(dX, M, K, code, dev, w + "dX")
    lddw = K if dWg is None else _pair(dWg, dWu, N, K, wcode, dev, (w + "dWg", w + "dWu"))
    d = GluBwdDesc(M, N, K, code, wcode, act, dH.data_ptr(), _matrix(dH, M, N, code, dev, w + "dH"), G.data_ptr(),
                   U.data_ptr(), _pair(G, U, M, N, code, dev, (w + "G", w + "U")), X.data_ptr(),
                   _matrix(X, M, K, code, dev, w + "X"), Wg.data_ptr(), Wu.data_ptr(),
                   _pair(Wg, Wu, N, K, code, dev, (w + "Wg", w + "Wu")), dx, lddx, _ptr(dWg), _ptr(dWu), lddw,
                   _vector(dbg, N, dev, w + "dbg"), _vector(dbu, N, dev, w + "dbu"), None, 0)
    _run(d, "structadmm_glu_bwd", lib().structadmm_glu_bwd_workspace, ws, X, stream)
    return dX, dWg, dWu, dbg, dbu


# ------------------------------------------------ 8-bit feed-forward operators
class Matrix8(NamedTuple):
    """An 8-bit matrix: codes [rows, cols] (float8_e4m3fn, or its bits as uint8) with rows
    on 16-byte boundaries, and float32 scales, one for each block of 128 columns of a row
    ([rows, ceil(cols / 128)]: "row blocks") or of 128 rows ([ceil(rows / 128), ..]: "square
    blocks")."""
    codes: "object"
    scales: "object"


def _blocks(n: int) -> int:
    return (n + BLOCK - 1) // BLOCK


def matrix8(rows: int, cols: int, block_rows: int = 1, device=None, stream=None) -> Matrix8:
    """An uninitialised 8-bit matrix as the calls below make them: rows of codes a
    multiple of 128 bytes apart, the scales of a block column side by side."""
    import torch
    if block_rows not in (1, BLOCK):
        raise StructAdmmError(f"matrix8: block_rows must be 1 or {BLOCK}, got {block_rows}")
    device = torch.device("cuda", torch.cuda.current_device()) if device is None else device
    nc, nr = _blocks(cols), rows if block_rows == 1 else _blocks(rows)
    codes = _empty(stream, (rows, nc * BLOCK), torch.uint8, device)
    scales = _empty(stream, (nc, nr), torch.float32, device)
    return Matrix8(codes.view(torch.float8_e4m3fn)[:, :cols], scales.t())


_e4m3 = []


def _matrix8(m, rows: int, cols: int, block_rows: int, dev, what: str) -> Matrix8Arg:
    """Checks a [rows, cols] 8-bit matrix argument (None: left out)."""
    if m is None:
        return Matrix8Arg(None, (cols + 15) // 16 * 16, None, 1, 1)
    if not _e4m3:
        import torch
        _e4m3.extend((torch.float8_e4m3fn, torch.uint8, torch.float32))
    codes, scales = m
    if codes.shape != (rows, cols) or codes.dtype not in _e4m3[:2]:
        raise StructAdmmError(f"{what} must hold e4m3 codes [{rows}, {cols}], got {codes.dtype} {tuple(codes.shape)}")
    nr, nc = rows if block_rows == 1 else _blocks(rows), _blocks(cols)
    if scales.shape != (nr, nc) or scales.dtype != _e4m3[2]:
        raise StructAdmmError(f"{what} must have float32 scales [{nr}, {nc}], got {scales.dtype} {tuple(scales.shape)}")
    if codes.device != dev or scales.device != dev:
        raise StructAdmmError(f"{what} is on {codes.device} and {scales.device}, not {dev}")
    ld, step = codes.stride()
    if step != 1 and cols > 1 and rows > 0:
        raise StructAdmmError(f"{what} must have unit column stride")
    if cols == 0 or rows <= 1 and (ld < cols or ld % 16 or ld > MAX_LD):
        ld = (cols + 15) // 16 * 16  # a single row has no pitch
    row, col = scales.stride()
    return Matrix8Arg(codes.data_ptr(), ld, scales.data_ptr(), row if nr > 1 and nc else 1, col if nc > 1 and nr else 1)


def _codes_of(m, what: str):
    """The [rows, cols] of an 8-bit operand in GPU memory."""
    if type(m) is not Matrix8 or m.codes.dim() != 2 or not m.codes.is_cuda:
        raise StructAdmmError(f"{what} must be a Matrix8 in GPU memory")
    if not _type_codes:
        _type_code(m.scales, what)
    return m.codes.shape


def rms_norm_fwd(X, gamma=None, R=None, eps: float = 1e-5, S=None, Y=None, Q=None, rstd=None, out: str = "ysr",
                 stream=None):
    """structadmm_rms_norm_fwd over the rows of S = X + R (X [rows, cols] bfloat16,
    float16 or float32; R like it or None); returns (Y, S, rstd, Q).  out names the
    outputs to make besides the buffers given: "y" (the result in X's type), "q" (in 8
    bits with row blocks), "s" (the sum; X itself where there is no R) and "r" (rstd,
    which the backward pass reads); the others are None."""
    import torch
    rows, cols = _rows_of(X, "rms_norm_fwd: X")
    dev, code, w = X.device, _type_code(X, "rms_norm_fwd: X"), "rms_norm_fwd: "
    if Y is None and "y" in out:
        Y = _new(stream, X, rows, cols)
    if S is None and R is not None and "s" in out:
        S = _new(stream, X, rows, cols)
    if Q is None and "q" in out:
        Q = matrix8(rows, cols, 1, dev, stream)
    if rstd is None and "r" in out:
        rstd = _empty(stream, rows, torch.float32, dev)
    r, ldr = _optional(R, rows, cols, code, dev, w + "R")
    s, lds = _optional(S, rows, cols, code, dev, w + "S")
    y, ldy = _optional(Y, rows, cols, code, dev, w + "Y")
    d = RmsNormDesc(rows, cols, code, eps, X.data_ptr(), _matrix(X, rows, cols, code, dev, w + "X"), r, ldr,
                    _vector(gamma, cols, dev, w + "gamma"), s, lds, y, ldy, _matrix8(Q, rows, cols, 1, dev, w + "Q"),
                    _vector(rstd, rows, dev, w + "rstd"))
    _run(d, "structadmm_rms_norm_fwd", None, None, X, stream)
    return Y, (X if S is None and R is None and "s" in out else S), rstd, Q


def rms_norm_bwd(dY, S, rstd, gamma=None, dR=None, dX=None, dgamma=None, params: bool = True, ws=None, stream=None):
    """structadmm_rms_norm_bwd; returns (dX, dgamma): dX is the gradient of X and of R.
    dR: the gradient that reaches S past the norm, added to dX.  dgamma is None with
    params=False (unless given)."""
    import torch
    rows, cols = _rows_of(S, "rms_norm_bwd: S")
    dev, code, w = S.device, _type_code(S, "rms_norm_bwd: S"), "rms_norm_bwd: "
    if rstd is None:
        raise StructAdmmError(w + "rstd of the forward pass is required")
    if dX is None:
        dX = _new(stream, S, rows, cols)
    if params and dgamma is None:
        dgamma = _empty(stream, cols, torch.float32, dev)
    r, ldr = _optional(dR, rows, cols, code, dev, w + "dR")
    d = RmsNormBwdDesc(rows, cols, code, dY.data_ptr(), _matrix(dY, rows, cols, code, dev, w + "dY"), S.data_ptr(),
                       _matrix(S, rows, cols, code, dev, w + "S"), _vector(rstd, rows, dev, w + "rstd"),
                       _vector(gamma, cols, dev, w + "gamma"), r, ldr, dX.data_ptr(),
                       _matrix(dX, rows, cols, code, dev, w + "dX"), _vector(dgamma, cols, dev, w + "dgamma"), None, 0)
    _run(d, "structadmm_rms_norm_bwd", lib().structadmm_rms_norm_bwd_workspace, ws, S, stream)
    return dX, dgamma


def quantize8(X, block_rows: int = 1, Q=None, QT=None, out: str = "q", stream=None):
    """structadmm_quantize8: X [rows, cols] (bfloat16, float16 or float32) in 8 bits, with
    row blocks (block_rows=1) or square blocks (128); returns (Q, QT).  out names what to
    make besides the matrices given: "q" (Q, as X stands) and "t" (QT [cols, rows], X
    transposed); the others are None."""
    rows, cols = _rows_of(X, "quantize8: X")
    dev, code, w = X.device, _type_code(X, "quantize8: X"), "quantize8: "
    if block_rows not in (1, BLOCK):
        raise StructAdmmError(f"{w}block_rows must be 1 or {BLOCK}, got {block_rows}")
    if Q is None and "q" in out:
        Q = matrix8(rows, cols, block_rows, dev, stream)
    if QT is None and "t" in out:
        QT = matrix8(cols, rows, block_rows, dev, stream)
    d = Quantize8Desc(rows, cols, code, block_rows, X.data_ptr(), _matrix(X, rows, cols, code, dev, w + "X"),
                      _matrix8(Q, rows, cols, block_rows, dev, w + "Q"),
                      _matrix8(QT, cols, rows, block_rows, dev, w + "QT"))
    _run(d, "structadmm_quantize8", None, None, X, stream)
    return Q, QT


def linear8_fwd(X, W, bias=None, R=None, act: int = ACT_NONE, Y=None, Z=None, Q=None, out_dtype=None, out: str = "y",
                ws=None, stream=None, exact: bool = False):
    """structadmm_linear8_fwd: act(X W^T + bias) + R for 8-bit X [M, K] (row blocks) and W
    [N, K] (square blocks); returns (Y, Q).  out names the results to make besides the
    buffers given: "y" (Y in out_dtype: R's type or else bfloat16 by default, float16 or
    float32) and "q" (Q in 8 bits with row blocks); the others are None.  R has Y's type.
    Z (bfloat16 or float16, Y's type unless that is float32): receives the
    pre-activations.  exact: whole products also where every result has 16 bits, whose
    sums may otherwise lose up to 2^-10 of their products' magnitudes (structadmm.h)."""
    import torch
    M, K = _codes_of(X, "linear8_fwd: X")
    N, _ = _codes_of(W, "linear8_fwd: W")
    dev, w = X[0].device, "linear8_fwd: "
    if Y is None and "y" in out:
        like = R.dtype if R is not None else torch.bfloat16 if Z is None else Z.dtype
        Y = _new(stream, X[0], M, N, out_dtype or like)
    if Q is None and "q" in out:
        Q = matrix8(M, N, 1, dev, stream)
    to = BF16 if Y is None and R is None else _type_code(R if Y is None else Y, w + "Y")
    code = _type_code(Z, w + "Z") if Z is not None else BF16 if to == F32 else to
    if Y is None and R is None:
        to = code
    r, ldr = _optional(R, M, N, to, dev, w + "R")
    y, ldy = _optional(Y, M, N, to, dev, w + "Y")
    z, ldz = _optional(Z, M, N, code, dev, w + "Z")
    d = Linear8Desc(M, N, K, code, to, act, _matrix8(X, M, K, 1, dev, w + "X"), _matrix8(W, N, K, BLOCK, dev, w + "W"),
                    _vector(bias, N, dev, w + "bias"), r, ldr, y, ldy, z, ldz, _matrix8(Q, M, N, 1, dev, w + "Q"), None, 0, exact)
    _run(d, "structadmm_linear8_fwd", lib().structadmm_linear8_workspace, ws, X[0], stream)
    return Y, Q


def glu8_fwd(X, Wg, Wu, bg=None, bu=None, act: int = ACT_SILU, H=None, Q=None, G=None, U=None, dtype=None,
             out: str = "q", ws=None, stream=None, exact: bool = False):
    """structadmm_glu8_fwd: act(X Wg^T + bg) * (X Wu^T + bu) for 8-bit X [M, K] (row blocks),
    Wg and Wu [N, K] (square blocks; one pitch and one layout of scales); returns (H, Q).
    out names the results to make besides the buffers given: "h" (H in dtype: G's type or
    else bfloat16 by default, or float16) and "q" (Q in 8 bits with row blocks); the others
    are None.  G and U (both or neither) receive the two projections, which glu_bwd reads.
    exact: as for linear8_fwd."""
    import torch
    M, K = _codes_of(X, "glu8_fwd: X")
    N, _ = _codes_of(Wg, "glu8_fwd: Wg")
    dev, w = X[0].device, "glu8_fwd: "
    if (G is None) != (U is None):
        raise StructAdmmError(w + "give both G and U or neither")
    if H is None and "h" in out:
        H = _new(stream, X[0], M, N, dtype or (torch.bfloat16 if G is None else G.dtype))
    if Q is None and "q" in out:
        Q = matrix8(M, N, 1, dev, stream)
    code = BF16 if H is None and G is None else _type_code(G if H is None else H, w + "H")
    h, ldh = _optional(H, M, N, code, dev, w + "H")
    ldgu = N if G is None else _pair(G, U, M, N, code, dev, (w + "G", w + "U"))
    d = Glu8Desc(M, N, K, code, act, _matrix8(X, M, K, 1, dev, w + "X"), _matrix8(Wg, N, K, BLOCK, dev, w + "Wg"),
                 _matrix8(Wu, N, K, BLOCK, dev, w + "Wu"), _vector(bg, N, dev, w + "bg"), _vector(bu, N, dev, w + "bu"),
                 h, ldh, _ptr(G), _ptr(U), ldgu, _matrix8(Q, M, N, 1, dev, w + "Q"), None, 0, exact)
    _run(d, "structadmm_glu8_fwd", lib().structadmm_glu8_workspace, ws, X[0], stream)
    return H, Q


def product8_plan(M: int, N: int, K: int, gated: bool = False, out: str = "y", f32: bool = False,
                  exact: bool = False) -> dict:
    """structadmm_linear8_plan (gated: structadmm_glu8_plan): the kernel that a product of
    these sizes takes for the outputs named in out ("y" or "h", "q"), host only.  f32: Y in
    float32.  "rows" (0: a tile of "tile_n" x "tile_m"), "exact", "split", "joined"."""
    info, at = Product8PlanInfo(), iter(range(1 << 12, 1 << 16, 1 << 8))  # addresses that nothing reads

    def m8(rows, cols, there=True):
        return Matrix8Arg(next(at) if there else None, (cols + 15) // 16 * 16, next(at) if there else None, 1, max(rows, 1))
    q, y = m8(M, N, "q" in out), next(at) if "y" in out or "h" in out else None
    x, w = m8(M, K), m8(_blocks(N), K)
    if gated:
        if f32:
            raise StructAdmmError("product8_plan: a gated product has no float32 result")
        d = Glu8Desc(M, N, K, BF16, ACT_NONE, x, w, w, None, None, y, N, None, None, N, q, None, 0, exact)
        _check(lib().structadmm_glu8_plan(ctypes.byref(d), ctypes.byref(info)), "structadmm_glu8_plan")
    else:
        d = Linear8Desc(M, N, K, BF16, F32 if f32 else BF16, ACT_NONE, x, w, None, None, N, y, N, None, N, q, None, 0, exact)
        _check(lib().structadmm_linear8_plan(ctypes.byref(d), ctypes.byref(info)), "structadmm_linear8_plan")
    return {n: getattr(info, n) for n, _ in Product8PlanInfo._fields_}


def version() -> str:
    return lib().structadmm_version().decode()

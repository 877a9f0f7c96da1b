"""Layer operators of n workers on 8-bit rows (the part of ``relaysum.h``
under that name): RMS norm with the residual's addition, products of packed
rows, their gradients, and packing.

Activations are CUDA tensors [n, tokens, width] in float32, bfloat16 or
float16, weights and weight gradients float32 views into the rows of the
models x[n, d] and the gradients g[n, d], for instance
``x[:, a:a + c * k].unflatten(1, (c, k))``.  Any strides will do as long as
the last axis is dense.  Results are new tensors, weight gradients go into
the tensor given for them.  Work is queued on torch's current stream.
"""
from __future__ import annotations

import ctypes
from typing import Optional

import torch

from . import RELAYSUM_OK, RelaySumError, _current_stream, load_library

RELAYSUM_FLOAT = 0
RELAYSUM_BFLOAT = 1
RELAYSUM_HALF = 2

TYPES = {torch.float32: RELAYSUM_FLOAT, torch.bfloat16: RELAYSUM_BFLOAT,
         torch.float16: RELAYSUM_HALF}
GROUP = 128
MAX_WIDTH = 32768


class Rows(ctypes.Structure):
    """struct relaysum_rows of relaysum.h."""
    _fields_ = [("data", ctypes.c_void_p), ("type", ctypes.c_int32),
                ("worker_stride", ctypes.c_int64), ("row_stride", ctypes.c_int64)]


class _CPacked(ctypes.Structure):
    """struct relaysum_packed of relaysum.h."""
    _fields_ = [("codes", ctypes.c_void_p), ("exps", ctypes.c_void_p), ("group", ctypes.c_int32)]


class Packed:
    """Packed rows of n workers: ``codes`` int8 [n, rows, stride] and ``exps``
    int8 [n, rows, groups], for rows of ``width`` entries; groups is 1 (whole
    rows share a scale) or stride / 128."""

    __slots__ = ("codes", "exps", "width")

    def __init__(self, codes, exps, width: int):
        self.codes, self.exps, self.width = codes, exps, int(width)
        n, rows, stride = codes.shape
        if stride != packed_stride(self.width):
            raise ValueError(f"rows of {self.width} entries have codes of stride "
                             f"{packed_stride(self.width)}, not {stride}")
        if exps.dim() != 3 or exps.shape[0] != n or exps.shape[1] != rows or \
                exps.shape[2] not in (1, stride // GROUP):
            raise ValueError(f"exps must have shape [{n}, {rows}, 1 or {stride // GROUP}]")
        for t, name in ((codes, "codes"), (exps, "exps")):
            if t.dtype != torch.int8 or not t.is_contiguous():
                raise ValueError(f"{name} must be a contiguous int8 tensor")
            _check_device(t, name)
        if codes.device != exps.device:
            raise ValueError("codes and exps must be on one device")

    @property
    def group(self) -> int:
        """128, or 0 for whole rows."""
        return 0 if self.exps.shape[2] == 1 else GROUP

    @property
    def shape(self):
        """(n, rows, width)."""
        return (*self.codes.shape[:2], self.width)

    def _c(self):
        return _CPacked(self.codes.data_ptr(), self.exps.data_ptr(), self.group)


def packed_stride(width: int) -> int:
    """Codes from the start of a packed row to the next."""
    if not 1 <= width <= MAX_WIDTH:
        raise ValueError(f"the width must be in 1..{MAX_WIDTH}")
    return -(-width // GROUP) * GROUP


_ready = None


def _lib():
    """The library with the signatures of this module's calls."""
    global _ready
    if _ready is None:
        lib = load_library()
        vp, i32, i64, sz = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_size_t
        rows, packed = ctypes.POINTER(Rows), ctypes.POINTER(_CPacked)
        sig = {
            "relaysum_packed_stride": (i64, [i64]),
            "relaysum_pack": (ctypes.c_int, [i32, i64, i64, rows, packed, vp]),
            "relaysum_unpack": (ctypes.c_int, [i32, i64, i64, packed, rows, vp]),
            "relaysum_rmsnorm": (ctypes.c_int, [i32, i64, i64, rows, rows, vp, i64, ctypes.c_float,
                                                rows, packed, vp, packed, vp]),
            "relaysum_rmsnorm_workspace": (i64, [i32, i64, i64]),
            "relaysum_rmsnorm_backward": (ctypes.c_int, [i32, i64, i64, rows, rows, packed, vp, vp,
                                                         i64, rows, rows, vp, sz, vp]),
            "relaysum_linear": (ctypes.c_int, [i32, i64, i64, i64, packed, packed, rows, vp, sz, vp]),
            "relaysum_linear_backward_input": (ctypes.c_int, [i32, i64, i64, i64, rows, packed,
                                                              rows, vp, sz, vp]),
            "relaysum_linear_workspace": (i64, [i32, i64, i64, i64, i32]),
            "relaysum_linear_backward_weight": (ctypes.c_int, [i32, i64, i64, i64, rows, packed,
                                                               rows, vp, sz, vp]),
            "relaysum_layer_error": (ctypes.c_char_p, []),
        }
        for name, (res, args) in sig.items():
            f = getattr(lib, name)
            f.restype, f.argtypes = res, args
        _ready = lib
    return _ready


def _check(rc: int, what: str) -> None:
    if rc != RELAYSUM_OK:
        raise RelaySumError(rc, f"{what} ({_lib().relaysum_layer_error().decode()})")


def _check_device(t, name: str) -> None:
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError(f"{name} must be a CUDA (HIP) tensor")
    if t.device.index != torch.cuda.current_device():
        raise ValueError(f"{name} must be on the current device")


def _rows(t, name: str, shape, dtype=None) -> Rows:
    """The description of a tensor [n, rows, width] (or [n, width]: one row
    for each worker) whose last axis is dense."""
    _check_device(t, name)
    if tuple(t.shape) != tuple(shape):
        raise ValueError(f"{name} must have shape {list(shape)}, not {list(t.shape)}")
    if t.dtype not in TYPES or (dtype is not None and t.dtype != dtype):
        want = dtype if dtype is not None else "float32, bfloat16 or float16"
        raise ValueError(f"{name} must be {want}, not {t.dtype}")
    st = t.stride()
    if t.shape[-1] > 1 and st[-1] != 1 and t.numel():
        raise ValueError(f"{name}: the last axis must be dense")
    return Rows(t.data_ptr(), TYPES[t.dtype], st[0], st[1] if len(st) == 3 else 0)


def _three(t, name: str):
    _check_device(t, name)
    if t.dim() != 3:
        raise ValueError(f"{name} must have three axes: workers, rows, width")
    return t.shape


def _new_packed(n: int, rows: int, width: int, group: int, device) -> Packed:
    stride = packed_stride(width)
    codes = torch.empty((n, rows, stride), dtype=torch.int8, device=device)
    exps = torch.empty((n, rows, stride // GROUP if group else 1), dtype=torch.int8, device=device)
    p = Packed.__new__(Packed)   # its parts fit by construction
    p.codes, p.exps, p.width = codes, exps, int(width)
    return p


def _workspace(nbytes: int, device):
    return torch.empty(nbytes, dtype=torch.uint8, device=device) if nbytes > 0 else None


def _ptr(t) -> Optional[int]:
    return None if t is None else t.data_ptr()


def pack(v, group: int = 0) -> Packed:
    """Rows v[n, rows, width] in 8 bits, one scale for each row (group 0) or
    for each 128 entries of it (group 128)."""
    n, rows, width = _three(v, "v")
    if group not in (0, GROUP):
        raise ValueError(f"group must be 0 or {GROUP}")
    r = _rows(v, "v", v.shape)
    out = _new_packed(n, rows, width, group, v.device)
    _check(_lib().relaysum_pack(n, rows, width, r, out._c(), _current_stream()), "relaysum_pack")
    return out


def unpack(p: Packed, dtype=torch.bfloat16):
    """The values of packed rows as a new tensor [n, rows, width]."""
    n, rows, width = p.shape
    if dtype not in TYPES:
        raise ValueError(f"dtype must be float32, bfloat16 or float16, not {dtype}")
    out = torch.empty((n, rows, width), dtype=dtype, device=p.codes.device)
    _check(_lib().relaysum_unpack(n, rows, width, p._c(), _rows(out, "out", out.shape),
                                  _current_stream()), "relaysum_unpack")
    return out


def rmsnorm(h, residual, weight, eps: float = 1e-6, keep: bool = True):
    """(sum, y, rstd, saved) with sum = h + residual, y = sum * rstd * weight
    packed by whole rows, rstd[n, tokens] = 1 / sqrt(mean(sum^2) + eps), and
    saved = sum packed by 128, for rmsnorm_backward (None without `keep`).
    weight[n, width]; residual may be None (sum is then h itself)."""
    n, tokens, width = _three(h, "h")
    rh = _rows(h, "h", h.shape)
    rw = _rows(weight, "weight", (n, width), torch.float32)
    out, rr, rs = h, None, None
    if residual is not None:
        rr = _rows(residual, "residual", h.shape, h.dtype)
        out = torch.empty((n, tokens, width), dtype=h.dtype, device=h.device)
        rs = _rows(out, "sum", out.shape)
    y = _new_packed(n, tokens, width, 0, h.device)
    saved = _new_packed(n, tokens, width, GROUP, h.device) if keep else None
    rstd = torch.empty((n, tokens), dtype=torch.float32, device=h.device)
    _check(_lib().relaysum_rmsnorm(n, tokens, width, rh, rr, rw.data, rw.worker_stride, float(eps),
                                   rs, y._c(), rstd.data_ptr(), saved._c() if keep else None,
                                   _current_stream()), "relaysum_rmsnorm")
    return out, y, rstd, saved


def rmsnorm_backward(dy, dsum, saved: Packed, rstd, weight, weight_grad):
    """The gradient of h and residual alike, as a new tensor, from the
    gradients dy of y and dsum of the sum (None: the sum is not used
    elsewhere); the weight's gradient overwrites weight_grad[n, width]."""
    n, tokens, width = _three(dy, "dy")
    rdy = _rows(dy, "dy", dy.shape)
    rd = None if dsum is None else _rows(dsum, "dsum", dy.shape, dy.dtype)
    if saved.shape != (n, tokens, width):
        raise ValueError(f"saved must hold rows [{n}, {tokens}, {width}], not {list(saved.shape)}")
    rw = _rows(weight, "weight", (n, width), torch.float32)
    rg = _rows(weight_grad, "weight_grad", (n, width), torch.float32)
    _rows(rstd, "rstd", (n, tokens), torch.float32)
    if not rstd.is_contiguous():
        raise ValueError("rstd must be contiguous")
    ds = torch.empty((n, tokens, width), dtype=dy.dtype, device=dy.device)
    lib = _lib()
    need = lib.relaysum_rmsnorm_workspace(n, tokens, width)
    ws = _workspace(need, dy.device)
    _check(lib.relaysum_rmsnorm_backward(n, tokens, width, rdy, rd, saved._c(), rstd.data_ptr(),
                                         rw.data, rw.worker_stride, _rows(ds, "ds", ds.shape), rg,
                                         _ptr(ws), max(need, 0), _current_stream()),
           "relaysum_rmsnorm_backward")
    return ds


def _same_width(x: Packed, w: Packed) -> None:
    if x.shape[0] != w.shape[0] or x.width != w.width:
        raise ValueError(f"packed rows of {list(x.shape)} and {list(w.shape)} do not go together")


def linear(x: Packed, w: Packed, dtype=torch.bfloat16):
    """y[n, tokens, channels] = x w^T of rows packed whole: tokens x[n, tokens,
    width], channels w[n, channels, width]."""
    _same_width(x, w)
    if dtype not in TYPES:
        raise ValueError(f"dtype must be float32, bfloat16 or float16, not {dtype}")
    n, tokens, width = x.shape
    channels = w.shape[1]
    y = torch.empty((n, tokens, channels), dtype=dtype, device=x.codes.device)
    lib = _lib()
    need = lib.relaysum_linear_workspace(n, tokens, width, channels, TYPES[dtype])
    ws = _workspace(need, y.device)
    _check(lib.relaysum_linear(n, tokens, width, channels, x._c(), w._c(), _rows(y, "y", y.shape),
                               _ptr(ws), max(need, 0), _current_stream()), "relaysum_linear")
    return y


def linear_backward_input(dy, w: Packed):
    """dx[n, tokens, width] = dy w, for dy[n, tokens, channels]."""
    n, tokens, channels = _three(dy, "dy")
    if w.shape[:2] != (n, channels):
        raise ValueError(f"dy of {list(dy.shape)} does not go with packed rows of {list(w.shape)}")
    rdy = _rows(dy, "dy", dy.shape)
    dx = torch.empty((n, tokens, w.width), dtype=dy.dtype, device=dy.device)
    lib = _lib()
    need = lib.relaysum_linear_workspace(n, tokens, w.width, channels, rdy.type)
    ws = _workspace(need, dy.device)
    _check(lib.relaysum_linear_backward_input(n, tokens, w.width, channels, rdy, w._c(),
                                              _rows(dx, "dx", dx.shape), _ptr(ws), max(need, 0),
                                              _current_stream()),
           "relaysum_linear_backward_input")
    return dx


def linear_backward_weight(dy, x: Packed, weight_grad) -> None:
    """weight_grad[n, channels, width] = dy^T x, for dy[n, tokens, channels]
    and packed x[n, tokens, width] of either group."""
    n, tokens, channels = _three(dy, "dy")
    if x.shape[:2] != (n, tokens):
        raise ValueError(f"dy of {list(dy.shape)} does not go with packed rows of {list(x.shape)}")
    rdy = _rows(dy, "dy", dy.shape)
    rg = _rows(weight_grad, "weight_grad", (n, channels, x.width), torch.float32)
    lib = _lib()
    need = lib.relaysum_linear_workspace(n, tokens, x.width, channels, rdy.type)
    ws = _workspace(need, dy.device)
    _check(lib.relaysum_linear_backward_weight(n, tokens, x.width, channels, rdy, x._c(), rg,
                                               _ptr(ws), max(need, 0), _current_stream()),
           "relaysum_linear_backward_weight")

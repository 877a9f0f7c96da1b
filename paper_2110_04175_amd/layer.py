"""Layer operators of n workers on 8-bit rows (the part of ``relaysum.h``
under that name): RMS norm with the residual's addition, products of packed
rows, their gradients, and packing.

Activations are CUDA tensors [n, tokens, width] in float32, bfloat16 or
float16, weights and weight gradients float32 views into the rows of the
models x[n, d] and the gradients g[n, d], for instance
``x[:, a:a + c * k].unflatten(1, (c, k))``.  Any strides will do as long as
the last axis is dense.  Results are new tensors, weight gradients go into
the tensor given for them.

Work is queued on torch's current stream; whoever uses a tensor, or the codes
and exps of a Packed, on another one orders the two and calls record_stream,
as for any tensor.  The operators take no part in autograd: results do not
require gradients whatever the inputs do, and a backward pass is made of the
``_backward`` calls (an autograd.Function can be built of them).
"""
from __future__ import annotations

import ctypes
import functools

import torch

from . import RELAYSUM_OK, RelaySumError, load_library

RELAYSUM_FLOAT = 0
RELAYSUM_BFLOAT = 1
RELAYSUM_HALF = 2

# relaysum_product
LINEAR = 0
LINEAR_BACKWARD_INPUT = 1
LINEAR_BACKWARD_WEIGHT = 2

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

    __slots__ = ("_codes", "_exps", "_buffer", "_n", "_rows", "_groups", "_device", "width")

    def __init__(self, codes, exps, width: int):
        stride = packed_stride(width)
        if not (isinstance(codes, torch.Tensor) and codes.is_cuda and isinstance(exps, torch.Tensor)
                and exps.is_cuda):
            raise TypeError("codes and exps must be CUDA (HIP) tensors")
        if codes.dtype != torch.int8 or exps.dtype != torch.int8 or codes.dim() != 3 or \
                not codes.is_contiguous() or not exps.is_contiguous():
            raise ValueError("codes and exps must be contiguous int8 tensors of three axes")
        n, rows, held = shape = codes.shape
        if held != stride:
            raise ValueError(f"rows of {width} entries have codes of stride {stride}, not {held}")
        groups = exps.shape[-1] if exps.dim() == 3 else 0
        if exps.shape[:-1] != shape[:-1] or (groups != 1 and groups != stride // GROUP):
            raise ValueError(f"exps must have shape [{n}, {rows}, 1 or {stride // GROUP}]")
        self._device = codes.get_device()
        if exps.get_device() != self._device:
            raise ValueError("codes and exps must be on one device")
        self._codes, self._exps, self._buffer = codes, exps, None
        self._n, self._rows, self._groups, self.width = n, rows, groups, width

    @classmethod
    def _new(cls, n: int, rows: int, width: int, group: int, like):
        """Room for packed rows, in one allocation: codes, then exponents."""
        p = cls.__new__(cls)
        stride = packed_stride(width)
        p._n, p._rows, p._groups, p.width = n, rows, stride // GROUP if group else 1, width
        p._codes = p._exps = None
        p._device = like.get_device()
        p._buffer = torch.empty(n * rows * (stride + p._groups), dtype=torch.int8, device=like.device)
        return p

    @property
    def stride(self) -> int:
        return -(-self.width // GROUP) * GROUP

    @property
    def codes(self):
        if self._codes is None:
            size = self._n * self._rows * self.stride
            self._codes = self._buffer[:size].view(self._n, self._rows, self.stride)
        return self._codes

    @property
    def exps(self):
        if self._exps is None:
            size = self._n * self._rows * self.stride
            self._exps = self._buffer[size:].view(self._n, self._rows, self._groups)
        return self._exps

    @property
    def group(self) -> int:
        """128, or 0 for whole rows."""
        return 0 if self._groups == 1 else GROUP

    @property
    def shape(self):
        """(n, rows, width)."""
        return (self._n, self._rows, self.width)

    def _c(self, device: int, name: str):
        if self._device != device:
            raise ValueError(f"{name} must be on the current device")
        group = 0 if self._groups == 1 else GROUP
        if self._buffer is not None:
            at = self._buffer.data_ptr()
            return _CPacked(at, at + self._n * self._rows * self.stride, group)
        return _CPacked(self._codes.data_ptr(), self._exps.data_ptr(), group)


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
            "relaysum_linear_workspace_of": (i64, [i32, i32, i64, i64, i64, i32]),
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


def _rows(t, name: str, shape, device: int, dtype=None) -> Rows:
    """The description of a tensor [n, rows, width] (or [n, width]: one row
    for each worker) whose last axis is dense."""
    if isinstance(t, torch.Tensor) and t.get_device() == device and t.shape == shape:
        code = TYPES.get(t.dtype)
        if code is not None and (dtype is None or t.dtype == dtype):
            st = t.stride()
            if st[-1] == 1 or shape[-1] <= 1 or not t.numel():
                return Rows(t.data_ptr(), code, st[0], st[1] if len(st) == 3 else 0)
    _refuse(t, name, shape, device, dtype)


def _refuse(t, name: str, shape, device: int, dtype) -> None:
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError(f"{name} must be a CUDA (HIP) tensor")
    if t.get_device() != device:
        raise ValueError(f"{name} must be on the current device")
    if t.shape != shape:
        raise ValueError(f"{name} must have shape {list(shape)}, not {list(t.shape)}")
    if t.dtype not in TYPES or (dtype is not None and t.dtype != dtype):
        want = dtype if dtype is not None else "float32, bfloat16 or float16"
        raise ValueError(f"{name} must be {want}, not {t.dtype}")
    raise ValueError(f"{name}: the last axis must be dense")


def _three(t, name: str):
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError(f"{name} must be a CUDA (HIP) tensor")
    if t.dim() != 3:
        raise ValueError(f"{name} must have three axes: workers, rows, width")
    return t.shape


def _out(n: int, rows: int, width: int, dtype, device):
    """(a new dense tensor [n, rows, width], its description)."""
    t = torch.empty((n, rows, width), dtype=dtype, device=device)
    return t, Rows(t.data_ptr(), TYPES[dtype], rows * width, width)


def _workspace(nbytes: int, device):
    """(address, bytes, what keeps it) of a workspace.  Memory of torch's
    allocator for the current stream, on which the call is queued too."""
    if nbytes <= 0:
        return None, 0, None
    t = torch.empty(nbytes, dtype=torch.uint8, device=device)
    return t.data_ptr(), nbytes, t


# A workspace's size follows from the call and its sizes alone.
@functools.lru_cache(maxsize=1024)
def _linear_workspace(product: int, n: int, tokens: int, width: int, channels: int, code: int) -> int:
    return _lib().relaysum_linear_workspace_of(product, n, tokens, width, channels, code)


@functools.lru_cache(maxsize=1024)
def _rmsnorm_workspace(n: int, tokens: int, width: int) -> int:
    return _lib().relaysum_rmsnorm_workspace(n, tokens, width)


def _here():
    """The current device and the address of its current stream."""
    device = torch.cuda.current_device()
    return device, torch._C._cuda_getCurrentRawStream(device)


def pack(v, group: int = 0) -> Packed:
    """Rows v[n, rows, width] in 8 bits, one scale for each row (group 0) or
    for each 128 entries of it (group 128)."""
    n, rows, width = shape = _three(v, "v")
    if group not in (0, GROUP):
        raise ValueError(f"group must be 0 or {GROUP}")
    device, stream = _here()
    r = _rows(v, "v", shape, device)
    out = Packed._new(n, rows, width, group, v)
    _check(_lib().relaysum_pack(n, rows, width, r, out._c(device, "out"), stream), "relaysum_pack")
    return out


def unpack(p: Packed, dtype=torch.bfloat16):
    """The values of packed rows as a new tensor [n, rows, width]."""
    n, rows, width = p.shape
    if dtype not in TYPES:
        raise ValueError(f"dtype must be float32, bfloat16 or float16, not {dtype}")
    device, stream = _here()
    cp = p._c(device, "p")
    out, ro = _out(n, rows, width, dtype, device)
    _check(_lib().relaysum_unpack(n, rows, width, cp, ro, stream), "relaysum_unpack")
    return out


def rmsnorm(h, residual, weight, eps: float = 1e-6, keep: bool = True):
    """(sum, y, rstd, saved) with sum = h + residual, y = sum * rstd * weight
    packed by whole rows, rstd[n, tokens] = 1 / sqrt(mean(sum^2) + eps), and
    saved = sum packed by 128, for rmsnorm_backward (None without `keep`).
    weight[n, width]; residual may be None (sum is then h itself)."""
    n, tokens, width = shape = _three(h, "h")
    device, stream = _here()
    rh = _rows(h, "h", shape, device)
    rw = _rows(weight, "weight", (n, width), device, torch.float32)
    out, rr, rs = h, None, None
    if residual is not None:
        rr = _rows(residual, "residual", shape, device, h.dtype)
        out, rs = _out(n, tokens, width, h.dtype, device)
    y = Packed._new(n, tokens, width, 0, h)
    saved = Packed._new(n, tokens, width, GROUP, h) if keep else None
    rstd = torch.empty((n, tokens), dtype=torch.float32, device=device)
    _check(_lib().relaysum_rmsnorm(n, tokens, width, rh, rr, rw.data, rw.worker_stride, eps, rs,
                                   y._c(device, "y"), rstd.data_ptr(),
                                   saved._c(device, "saved") if keep else None, stream),
           "relaysum_rmsnorm")
    return out, y, rstd, saved


def rmsnorm_backward(dy, dsum, saved: Packed, rstd, weight, weight_grad):
    """The gradient of h and residual alike, as a new tensor, from the
    gradients dy of y and dsum of the sum (None: the sum is not used
    elsewhere); the weight's gradient overwrites weight_grad[n, width]."""
    n, tokens, width = shape = _three(dy, "dy")
    device, stream = _here()
    rdy = _rows(dy, "dy", shape, device)
    rd = None if dsum is None else _rows(dsum, "dsum", shape, device, dy.dtype)
    if saved.shape != (n, tokens, width):
        raise ValueError(f"saved must hold rows [{n}, {tokens}, {width}], not {list(saved.shape)}")
    rw = _rows(weight, "weight", (n, width), device, torch.float32)
    rg = _rows(weight_grad, "weight_grad", (n, width), device, torch.float32)
    _rows(rstd, "rstd", (n, tokens), device, torch.float32)
    if not rstd.is_contiguous():
        raise ValueError("rstd must be contiguous")
    ds, rs = _out(n, tokens, width, dy.dtype, device)
    lib = _lib()
    ws, size, _keep = _workspace(_rmsnorm_workspace(n, tokens, width), device)
    _check(lib.relaysum_rmsnorm_backward(n, tokens, width, rdy, rd, saved._c(device, "saved"),
                                         rstd.data_ptr(), rw.data, rw.worker_stride, rs, rg, ws,
                                         size, stream), "relaysum_rmsnorm_backward")
    return ds


def linear(x: Packed, w: Packed, dtype=torch.bfloat16):
    """y[n, tokens, channels] = x w^T of rows packed whole: tokens x[n, tokens,
    width], channels w[n, channels, width]."""
    n, tokens, width = x.shape
    if w.shape[0] != n or w.width != width:
        raise ValueError(f"packed rows of {list(x.shape)} and {list(w.shape)} do not go together")
    if dtype not in TYPES:
        raise ValueError(f"dtype must be float32, bfloat16 or float16, not {dtype}")
    channels = w.shape[1]
    device, stream = _here()
    cx, cw = x._c(device, "x"), w._c(device, "w")
    y, ry = _out(n, tokens, channels, dtype, device)
    lib = _lib()
    ws, size, _keep = _workspace(_linear_workspace(LINEAR, n, tokens, width, channels, ry.type), device)
    _check(lib.relaysum_linear(n, tokens, width, channels, cx, cw, ry, ws, size, stream),
           "relaysum_linear")
    return y


def linear_backward_input(dy, w: Packed):
    """dx[n, tokens, width] = dy w, for dy[n, tokens, channels]."""
    n, tokens, channels = shape = _three(dy, "dy")
    if w.shape[:2] != (n, channels):
        raise ValueError(f"dy of {list(shape)} does not go with packed rows of {list(w.shape)}")
    width = w.width
    device, stream = _here()
    rdy, cw = _rows(dy, "dy", shape, device), w._c(device, "w")
    dx, rdx = _out(n, tokens, width, dy.dtype, device)
    lib = _lib()
    ws, size, _keep = _workspace(_linear_workspace(LINEAR_BACKWARD_INPUT, n, tokens, width, channels, rdy.type), device)
    _check(lib.relaysum_linear_backward_input(n, tokens, width, channels, rdy, cw, rdx, ws, size,
                                              stream), "relaysum_linear_backward_input")
    return dx


def linear_backward_weight(dy, x: Packed, weight_grad) -> None:
    """weight_grad[n, channels, width] = dy^T x, for dy[n, tokens, channels]
    and packed x[n, tokens, width] of either group."""
    n, tokens, channels = shape = _three(dy, "dy")
    if x.shape[:2] != (n, tokens):
        raise ValueError(f"dy of {list(shape)} does not go with packed rows of {list(x.shape)}")
    width = x.width
    device, stream = _here()
    rdy, cx = _rows(dy, "dy", shape, device), x._c(device, "x")
    rg = _rows(weight_grad, "weight_grad", (n, channels, width), device, torch.float32)
    lib = _lib()
    ws, size, _keep = _workspace(_linear_workspace(LINEAR_BACKWARD_WEIGHT, n, tokens, width, channels, rdy.type), device)
    _check(lib.relaysum_linear_backward_weight(n, tokens, width, channels, rdy, cx, rg, ws, size,
                                               stream), "relaysum_linear_backward_weight")

"""Binding of the 8-bit operators of ``include/vp.h``: matrices held in e4m3
with a power of two for each block of 128 columns, their products, and the
root-mean-square norm with its gradients.

As in the rest of the binding, the ``vp_*`` functions take the caller's
buffers and a stream; the others allocate their outputs with torch and run on
the current stream.  Nothing here computes: every call is one native entry.
Dense matrices are CUDA tensors [rows, cols] of float32 or bfloat16 whose rows
are contiguous (any distance between rows).

No function records a graph for torch.autograd: the gradients are calls of
their own.  A forward call on a tensor that requires a gradient, where
gradients are being recorded, is refused; under torch.no_grad(), and so in the
forward method of a torch.autograd.Function, it is not.
"""
from __future__ import annotations

import ctypes
import functools

import numpy as np
import torch

from . import VP_ERR_ARG, VP_ERR_DIMS, VP_OK, VP_OUT_BF16, VP_OUT_F32, VPError, _check, _stream_handle, lib

VP_MAX_DIM = 0x7fffff00
VP_MAX_SUM = 0x3ffff80
VP_PRODUCT_TILES, VP_PRODUCT_WAVES, VP_PRODUCT_JOIN = 0, 1, 2
_TYPES = {torch.float32: VP_OUT_F32, torch.bfloat16: VP_OUT_BF16}
_NAMES = {"bf16": torch.bfloat16, "f32": torch.float32, torch.bfloat16: torch.bfloat16, torch.float32: torch.float32}
_Q = torch.float8_e4m3fn
_stream_of = torch._C._cuda_getCurrentRawStream if hasattr(torch._C, "_cuda_getCurrentRawStream") else None


class vp_fp8(ctypes.Structure):
    _fields_ = [("q", ctypes.c_void_p), ("scale", ctypes.c_void_p), ("rows", ctypes.c_int64),
                ("cols", ctypes.c_int64), ("block", ctypes.c_int32), ("reserved", ctypes.c_int32)]


_fp8p = ctypes.POINTER(vp_fp8)
_i32, _i64, _p, _f32 = ctypes.c_int32, ctypes.c_int64, ctypes.c_void_p, ctypes.c_float
ARGTYPES = {
    "vp_fp8_layout": [_i64, _i64, _i32, ctypes.POINTER(_i64), ctypes.POINTER(_i64)],
    "vp_fp8_quantize": [_p, _i32, _i64, _i64, _i64, _fp8p, _fp8p, _p],
    "vp_fp8_transpose": [_fp8p, _fp8p, _p],
    "vp_fp8_dequantize": [_fp8p, _p, _i32, _i64, _p],
    "vp_fp8_matmul_workspace": [_i64, _i64, _i64, _i32, ctypes.POINTER(_i64)],
    "vp_fp8_matmul": [_fp8p, _fp8p, _p, _i32, _i64, _p, _i64, _p],
    "vp_fp8_matmul_kernels": [_i64, _i64, _i64, _i32, _i64, ctypes.POINTER(_i32), _i32, ctypes.POINTER(_i32)],
    "vp_rms_norm": [_p, _i64, _p, _i64, _p, _i32, _i64, _i64, _f32, _p, _i64, _p, _i64, _fp8p, _p, _p],
    "vp_rms_norm_backward_workspace": [_i64, _i64, ctypes.POINTER(_i64)],
    "vp_rms_norm_backward": [_p, _i64, _p, _i64, _p, _p, _p, _i64, _i32, _i64, _i64, _p, _i64, _p, _p, _i64, _p],
}


class _Entries:
    """The native functions, looked up once each."""

    def __getattr__(self, name: str):
        f = getattr(lib(), name)
        f.argtypes, f.restype = ARGTYPES[name], _i32
        setattr(self, name, f)
        return f


_native = _Entries()


def _entry(name: str):
    return getattr(_native, name)


def _bad(message: str, status: int = VP_ERR_ARG):
    raise VPError(status, message)


class Fp8:
    """A matrix [rows, cols] held in 8 bits.

    q: float8_e4m3fn [rows, cols rounded up to 128], zero beyond cols; scale:
    uint8 [rows or ceil(rows / 128), ceil(cols / 128) rounded up to 4], a byte
    b >= 1 for 2^(b - 127) (255: not a number).  block: 1 (a scale for each row and
    128 columns: activations, gradients) or 128 (for each 128 x 128: weights).
    """
    # Matrices that the operators allocate are one buffer (an allocation costs
    # the host as much as a third of a launch); their tensors are views made
    # when someone asks for them.
    __slots__ = ("rows", "cols", "block", "_c", "_device", "_q", "_scale", "_buffer")

    def __init__(self, q, scale, cols: int, block: int = 1):
        device = q.get_device()
        if q.dtype is not _Q or scale.dtype is not torch.uint8 or device < 0 or scale.get_device() != device \
                or q.dim() != 2 or scale.dim() != 2 or not q.is_contiguous() or not scale.is_contiguous():
            _bad("q must be a contiguous CUDA float8_e4m3fn matrix and scale a contiguous uint8 one beside it")
        rows, ld = q.shape
        groups, sld = scale.shape
        if block != 1 and block != 128:
            _bad("block must be 1 or 128")
        if cols < 0 or ld != -(-cols // 128) * 128 or sld != -(-cols // 512) * 4 or groups != -(-rows // block):
            _bad(f"q {tuple(q.shape)} and scale {tuple(scale.shape)} do not fit {cols} columns in blocks of "
                 f"{block} x 128", VP_ERR_DIMS)
        self.rows, self.cols, self.block, self._device = rows, cols, block, device
        self._q, self._scale, self._buffer = q, scale, None
        self._c = vp_fp8(q.data_ptr(), scale.data_ptr(), rows, cols, block, 0)

    @classmethod
    def empty(cls, rows: int, cols: int, block: int = 1, device=None) -> "Fp8":
        """Buffers for a matrix, uninitialised."""
        if block != 1 and block != 128:
            _bad("block must be 1 or 128")
        if not 0 <= rows <= VP_MAX_DIM or not 0 <= cols <= VP_MAX_DIM:
            _bad("rows and cols must lie in [0, VP_MAX_DIM]", VP_ERR_DIMS)
        size = rows * (-(-cols // 128) * 128)
        buffer = torch.empty(size + -(-rows // block) * (-(-cols // 512) * 4), dtype=torch.uint8,
                             device="cuda" if device is None else device)
        self = cls.__new__(cls)
        self.rows, self.cols, self.block, self._device = rows, cols, block, buffer.get_device()
        self._q, self._scale, self._buffer = None, None, buffer
        at = buffer.data_ptr()
        self._c = vp_fp8(at, at + size, rows, cols, block, 0)
        return self

    @property
    def q(self):
        if self._q is None:
            ld = -(-self.cols // 128) * 128
            self._q = self._buffer[:self.rows * ld].view(_Q).view(self.rows, ld)
        return self._q

    @property
    def scale(self):
        if self._scale is None:
            size = self.rows * (-(-self.cols // 128) * 128)
            self._scale = self._buffer[size:].view(-(-self.rows // self.block), -(-self.cols // 512) * 4)
        return self._scale

    @property
    def shape(self):
        return self.rows, self.cols

    @property
    def device(self):
        return (self._buffer if self._q is None else self._q).device

    def record_stream(self, stream):
        """As torch.Tensor.record_stream: the memory is in use on `stream` too."""
        for t in (self._buffer, self._q, self._scale):
            if t is not None:
                t.record_stream(stream)

    def __repr__(self):
        return f"Fp8({self.rows} x {self.cols}, block {self.block}, {self.device})"


def _dense(t, name: str, dtype=None, rows=None, cols=None):
    """(pointer, distance between rows) of a dense matrix argument."""
    if t.dtype not in _TYPES or not t.is_cuda or t.dim() != 2:
        _bad(f"{name} must be a CUDA matrix of float32 or bfloat16")
    r, c = t.shape
    if dtype is not None and t.dtype is not dtype:
        _bad(f"{name} must be of {dtype}")
    if (rows is not None and r != rows) or (cols is not None and c != cols):
        _bad(f"{name} is {tuple(t.shape)}, and ({rows}, {cols}) is needed", VP_ERR_DIMS)
    ld, one = t.stride()
    if one != 1 and c > 1:
        _bad(f"the rows of {name} must be contiguous")
    if r <= 1 and ld < c:
        ld = c
    return t.data_ptr(), ld


def _vector(t, name: str, dtype, n: int):
    if t.dtype is not dtype or not t.is_cuda or t.dim() != 1 or not t.is_contiguous():
        _bad(f"{name} must be a contiguous CUDA vector of {dtype}")
    if t.shape[0] != n:
        _bad(f"{name} holds {t.shape[0]} values, and {n} are needed", VP_ERR_DIMS)
    return t.data_ptr()


def _no_graph(*tensors):
    """Refuses what a graph would have to be recorded for."""
    if torch.is_grad_enabled():
        for t in tensors:
            if t is not None and t.requires_grad:
                _bad("a tensor requires a gradient, and no graph is recorded here: call under torch.no_grad() (the gradients "
                     "are calls of their own) or on its detach()")


def _same_device(device: int, *others):
    """Every tensor on the current device, where the kernels run."""
    if device != torch._C._cuda_getDevice():
        _bad("the tensors must be on the current device")
    for t in others:
        if t is not None and (t._device if t.__class__ is Fp8 else t.get_device()) != device:
            _bad("the tensors must be on one device")
    return device


def _stream(stream, device: int):
    if stream is None and _stream_of is not None:
        return _stream_of(device)
    return _stream_handle(stream)


def _workspace(t):
    if t is None:
        return 0, 0
    if not t.is_cuda or not t.is_contiguous():
        _bad("workspace must be a contiguous CUDA tensor")
    return t.data_ptr(), t.numel() * t.element_size()


# --------------------------------------------------------------------------
# The native entries on the caller's buffers
# --------------------------------------------------------------------------

def vp_fp8_layout(rows: int, cols: int, block: int = 1):
    """(bytes of q, bytes of scale)."""
    q, s = _i64(), _i64()
    _check(_native.vp_fp8_layout(rows, cols, block, ctypes.byref(q), ctypes.byref(s)), "vp_fp8_layout")
    return q.value, s.value


def vp_fp8_quantize(x, by_rows=None, by_cols=None, stream=None):
    """x [rows, cols] into 8 bits: by_rows Fp8 [rows, cols] and / or by_cols Fp8 [cols, rows], the transpose."""
    _no_graph(x)
    ptr, ld = _dense(x, "x")
    device = _same_device(x.get_device(), by_rows, by_cols)
    rows, cols = x.shape
    st = _native.vp_fp8_quantize(ptr, _TYPES[x.dtype], rows, cols, ld, by_rows and by_rows._c, by_cols and by_cols._c,
                                 _stream(stream, device))
    if st:
        _check(st, "vp_fp8_quantize")


def vp_fp8_transpose(src: Fp8, out: Fp8, stream=None):
    """out [cols, rows] = the transpose of src [rows, cols], blocks along the other axis."""
    st = _native.vp_fp8_transpose(src._c, out._c, _stream(stream, _same_device(src._device, out)))
    if st:
        _check(st, "vp_fp8_transpose")


def vp_fp8_dequantize(src: Fp8, out, stream=None):
    """out [rows, cols] = the values of src."""
    ptr, ld = _dense(out, "out", None, src.rows, src.cols)
    st = _native.vp_fp8_dequantize(src._c, ptr, _TYPES[out.dtype], ld, _stream(stream, _same_device(src._device, out)))
    if st:
        _check(st, "vp_fp8_dequantize")


@functools.lru_cache(maxsize=4096)
def vp_fp8_matmul_workspace(m: int, n: int, k: int, out_dtype: int = VP_OUT_BF16) -> int:
    """Bytes of workspace of vp_fp8_matmul, a function of the sizes alone."""
    b = _i64()
    _check(_native.vp_fp8_matmul_workspace(m, n, k, out_dtype, ctypes.byref(b)), "vp_fp8_matmul_workspace")
    return b.value


def vp_fp8_matmul(a: Fp8, b: Fp8, out, workspace=None, stream=None):
    """out [M, N] = a [M, K] b [N, K]^T, in out's type."""
    ptr, ld = _dense(out, "out", None, a.rows, b.rows)
    work, size = _workspace(workspace)
    st = _native.vp_fp8_matmul(a._c, b._c, ptr, _TYPES[out.dtype], ld, work, size,
                               _stream(stream, _same_device(a._device, b, out, workspace)))
    if st:
        _check(st, "vp_fp8_matmul")


def vp_fp8_matmul_kernels(m: int, n: int, k: int, out_dtype: int = VP_OUT_BF16, ld=None):
    """The launches vp_fp8_matmul makes for these sizes, as int32 rows (kind, tile rows, tile columns, pieces of the sum);
    no kernel runs."""
    rows, count = (_i32 * 8)(), _i32()
    _check(_native.vp_fp8_matmul_kernels(m, n, k, out_dtype, n if ld is None else ld, rows, 2, ctypes.byref(count)),
           "vp_fp8_matmul_kernels")
    return np.array(rows, np.int32).reshape(2, 4)[:count.value]


def vp_rms_norm(x, weight, residual=None, eps: float = 1e-6, h=None, out=None, out8=None, rstd=None, stream=None):
    """h = x + residual, out / out8 = h * rstd * weight, rstd = 1 / sqrt(mean(h^2) + eps); outputs that are None
    are not written."""
    _no_graph(x, weight, residual)
    px, ldx = _dense(x, "x")
    dtype = x.dtype
    rows, cols = x.shape
    pr, ldr = (0, 0) if residual is None else _dense(residual, "residual", dtype, rows, cols)
    ph, ldh = (0, 0) if h is None else _dense(h, "h", dtype, rows, cols)
    po, ldo = (0, 0) if out is None else _dense(out, "out", dtype, rows, cols)
    ps = 0 if rstd is None else _vector(rstd, "rstd", torch.float32, rows)
    pw = _vector(weight, "weight", dtype, cols)
    device = _same_device(x.get_device(), weight, residual, h, out, out8, rstd)
    st = _native.vp_rms_norm(px, ldx, pr, ldr, pw, _TYPES[dtype], rows, cols, eps, ph, ldh, po, ldo, out8 and out8._c,
                             ps, _stream(stream, device))
    if st:
        _check(st, "vp_rms_norm")


@functools.lru_cache(maxsize=4096)
def vp_rms_norm_backward_workspace(rows: int, cols: int) -> int:
    """Bytes of workspace of vp_rms_norm_backward with dweight, a function of the sizes alone."""
    b = _i64()
    _check(_native.vp_rms_norm_backward_workspace(rows, cols, ctypes.byref(b)), "vp_rms_norm_backward_workspace")
    return b.value


def vp_rms_norm_backward(dy, h, weight, rstd, dx, dweight=None, dh=None, workspace=None, stream=None):
    """dx (for x and the residual alike) and, unless None, dweight; dh: the gradient that reaches h by the skip path."""
    ph, ldh = _dense(h, "h")
    dtype = h.dtype
    rows, cols = h.shape
    py, ldy = _dense(dy, "dy", dtype, rows, cols)
    pd, lddh = (0, 0) if dh is None else _dense(dh, "dh", dtype, rows, cols)
    px, lddx = _dense(dx, "dx", dtype, rows, cols)
    pw = _vector(weight, "weight", dtype, cols)
    ps = _vector(rstd, "rstd", torch.float32, rows)
    pg = 0 if dweight is None else _vector(dweight, "dweight", torch.float32, cols)
    work, size = _workspace(workspace)
    device = _same_device(h.get_device(), dy, weight, rstd, dh, dx, dweight, workspace)
    st = _native.vp_rms_norm_backward(py, ldy, ph, ldh, pw, ps, pd, lddh, _TYPES[dtype], rows, cols, px, lddx, pg,
                                      work, size, _stream(stream, device))
    if st:
        _check(st, "vp_rms_norm_backward")


# --------------------------------------------------------------------------
# With outputs from torch, on the current stream.  What these allocate needs
# no checks, so the short ones go to the native entry directly.
# --------------------------------------------------------------------------

def _dtype(name):
    t = _NAMES.get(name)
    return t if t is not None else _bad(f"unknown element type {name!r}: bf16 or f32")


def fp8_quantize(x, block: int = 1, rows: bool = True, cols: bool = False):
    """x [M, K] in 8 bits: as it lies (rows), transposed (cols: Fp8 [K, M], blocks along M), or both, as a pair."""
    if not (rows or cols):
        _bad("neither rows nor cols")
    _no_graph(x)
    ptr, ld = _dense(x, "x")
    m, k = x.shape
    device = _same_device(x.get_device())
    a = Fp8.empty(m, k, block, x.device) if rows else None
    b = Fp8.empty(k, m, block, x.device) if cols else None
    st = _native.vp_fp8_quantize(ptr, _TYPES[x.dtype], m, k, ld, a and a._c, b and b._c, _stream(None, device))
    if st:
        _check(st, "vp_fp8_quantize")
    return (a, b) if rows and cols else a if rows else b


def fp8_transpose(src: Fp8) -> Fp8:
    """The transpose in 8 bits: of a weight (block 128) exactly; of a checkpoint of activations (block 1) with its
    blocks along the rows, as the product for the weight's gradient reads it."""
    out = Fp8.empty(src.cols, src.rows, src.block, src.device)
    vp_fp8_transpose(src, out)
    return out


def fp8_dequantize(src: Fp8, out_dtype="bf16"):
    """The values of src, [rows, cols] in bf16 or f32."""
    dtype = _dtype(out_dtype)
    device = _same_device(src._device)
    out = torch.empty(src.rows, src.cols, dtype=dtype, device=src.device)
    st = _native.vp_fp8_dequantize(src._c, out.data_ptr(), _TYPES[dtype], src.cols, _stream(None, device))
    if st:
        _check(st, "vp_fp8_dequantize")
    return out


def fp8_matmul(a: Fp8, b: Fp8, out_dtype="bf16"):
    """a [M, K] b [N, K]^T in bf16 or f32.  A linear layer: y = fp8_matmul(x, w); its gradients: dx =
    fp8_matmul(dy, fp8_transpose(w)), dw = fp8_matmul(dy_t, fp8_transpose(x), "f32") with
    dy, dy_t = fp8_quantize(grad, cols=True).  Results in f32 have sums in f32; those in bf16 are formed by the 8-bit
    instructions, which lose the products below 2^-13 of the largest of 8 neighbours: fp8_matmul(a, b, "f32").bfloat16()
    does not."""
    dtype = _dtype(out_dtype)
    device = _same_device(a._device, b)
    m, n, code, where = a.rows, b.rows, _TYPES[dtype], a.device
    size = vp_fp8_matmul_workspace(m, n, a.cols, code)
    out = torch.empty(m, n, dtype=dtype, device=where)
    work = torch.empty(size, dtype=torch.uint8, device=where) if size else None   # held until the call has enqueued
    st = _native.vp_fp8_matmul(a._c, b._c, out.data_ptr(), code, n, work.data_ptr() if size else 0, size,
                               _stream(None, device))
    if st:
        _check(st, "vp_fp8_matmul")
    return out


def rms_norm(x, weight, residual=None, eps: float = 1e-6, out=None):
    """(y, h, rstd): h = x + residual (x itself without one), y = h * rstd * weight, in x's type, or with out="fp8"
    as an Fp8 that fp8_matmul takes."""
    if out not in (None, "fp8"):
        _bad(f"unknown output {out!r}: None (x's type) or 'fp8'")
    _no_graph(x, weight, residual)
    px, ldx = _dense(x, "x")
    dtype, where = x.dtype, x.device
    rows, cols = x.shape
    pw = _vector(weight, "weight", dtype, cols)
    device = _same_device(x.get_device(), weight, residual)
    if residual is None:
        pr, ldr, h, ph = 0, 0, x, 0
    else:
        pr, ldr = _dense(residual, "residual", dtype, rows, cols)
        h = torch.empty(rows, cols, dtype=dtype, device=where)
        ph = h.data_ptr()
    rstd = torch.empty(rows, dtype=torch.float32, device=where)
    if out is None:
        y = torch.empty(rows, cols, dtype=dtype, device=where)
        po, p8 = y.data_ptr(), None
    else:
        y = Fp8.empty(rows, cols, 1, where)
        po, p8 = 0, y._c
    st = _native.vp_rms_norm(px, ldx, pr, ldr, pw, _TYPES[dtype], rows, cols, eps, ph, cols, po, cols, p8,
                             rstd.data_ptr(), _stream(None, device))
    if st:
        _check(st, "vp_rms_norm")
    return y, h, rstd


def rms_norm_backward(dy, h, weight, rstd, dh=None):
    """(dx, dweight f32) of rms_norm, from the h and rstd that it returned; dx is the gradient of x and of the residual."""
    ph, ldh = _dense(h, "h")
    dtype, where = h.dtype, h.device
    rows, cols = h.shape
    py, ldy = _dense(dy, "dy", dtype, rows, cols)
    pd, lddh = (0, 0) if dh is None else _dense(dh, "dh", dtype, rows, cols)
    pw, ps = _vector(weight, "weight", dtype, cols), _vector(rstd, "rstd", torch.float32, rows)
    device = _same_device(h.get_device(), dy, weight, rstd, dh)
    dx = torch.empty(rows, cols, dtype=dtype, device=where)
    dweight = torch.empty(cols, dtype=torch.float32, device=where)
    size = vp_rms_norm_backward_workspace(rows, cols)
    work = torch.empty(size, dtype=torch.uint8, device=where)   # held until the call is enqueued
    st = _native.vp_rms_norm_backward(py, ldy, ph, ldh, pw, ps, pd, lddh, _TYPES[dtype], rows, cols, dx.data_ptr(),
                                      cols, dweight.data_ptr(), work.data_ptr(), size, _stream(None, device))
    if st:
        _check(st, "vp_rms_norm_backward")
    return dx, dweight

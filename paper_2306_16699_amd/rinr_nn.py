"""ctypes binding of include/rinr_nn.h: operators for the network that learns from decoded batches.

Argument marshalling only; every operator runs in the HIP kernels of librinr.so.  PyTorch owns memory and streams.  Activations are matrices
whose last dimension has unit stride (any leading dimensions that lie evenly apart); weights are [n_out, n_in]; bias and gain are
float32.  `stream`: a torch stream, an integer handle (0: the GPU's default stream) or None for the current one; outputs and scratch
memory come from the stream that works on them.  What the caller passes has to be ready there; it may be dropped at once, as its memory is not handed
on before that stream has done with it.

No operator keeps a graph for automatic differentiation: while gradients are being recorded, tensors that require them are refused.  Under torch.no_grad(),
and so inside the forward and backward of a torch.autograd.Function, whose gradients are those of the `_backward` operators, they are taken.
"""
from __future__ import annotations

import ctypes as C
import math
import struct
from typing import Optional

import torch

from . import rinr

EXPORTS = ["rinr_linear_workspace_bytes", "rinr_linear", "rinr_linear_backward_workspace_bytes", "rinr_linear_backward", "rinr_rms_norm",
           "rinr_rms_norm_backward_workspace_bytes", "rinr_rms_norm_backward", "rinr_pack8", "rinr_unpack8"]
TYPES = {torch.bfloat16: 1, torch.float16: 2, torch.float32: 3}
PACKED8 = 4
ACTS = {"none": 0, "relu": 1, "gelu": 2, "silu": 3, "sine": 4}
BLOCK = 32                       # columns of a row that share a scale
MAX_NORM_COLS = 32768
# The argument structures of the header as bytes: a ctypes.Structure of as many fields takes several microseconds to fill
_LINEAR = struct.Struct("=qqq PqP Pq P Pq Pq PqP iiiifi".replace(" ", "").replace("P", "Q"))
_LINEAR_GRAD = struct.Struct("=qqqQqQqQQqQqQQqQqQiiiiif")
_NORM = struct.Struct("=qqQqQqQQqQQqiifi")
_NORM_GRAD = struct.Struct("=qqQqQqQQqQqQif")

_lib = None


def lib():
    global _lib
    if _lib is None:
        L = rinr.lib()
        vp, i32, i64, sz, f32 = C.c_void_p, C.c_int32, C.c_int64, C.c_size_t, C.c_float
        for name in ("rinr_linear_workspace_bytes", "rinr_linear_backward_workspace_bytes"):
            getattr(L, name).argtypes = [C.c_char_p]
            getattr(L, name).restype = sz
        L.rinr_linear.argtypes = L.rinr_linear_backward.argtypes = L.rinr_rms_norm_backward.argtypes = [C.c_char_p, vp, sz, vp]
        L.rinr_rms_norm.argtypes = [C.c_char_p, vp]
        L.rinr_rms_norm_backward_workspace_bytes.argtypes = [i64, i64]
        L.rinr_rms_norm_backward_workspace_bytes.restype = sz
        L.rinr_pack8.argtypes = [i64, i64, vp, i64, i32, vp, i64, vp, vp]
        L.rinr_unpack8.argtypes = [i64, i64, vp, i64, vp, i32, f32, vp, i64, i32, vp]
        _lib = L
    return _lib


def _require(ok: bool, what: str):
    if not ok:
        raise rinr.RinrError(rinr.E_ARG, what)


class Packed8:
    """A matrix in 8 bits: codes int8 [rows, whole blocks of 32 columns], scales uint8 [rows, blocks], and how many columns there are;
    the value is code * 2^(scale - 127).  `shape` is that of the tensor it stands for: any leading dimensions of `rows` rows in all, and the
    columns.  What a Packed8 says of itself cannot be set: results are allocated by it."""
    __slots__ = ("_codes", "_scales", "_both", "_rows", "_cols", "_ld", "_shape", "_device")

    def __init__(self, codes, scales, cols: int, shape=None):
        _require(codes.dtype == torch.int8 and scales.dtype == torch.uint8 and codes.dim() == 2 and cols >= 1, "Packed8: int8 codes, uint8 scales")
        rows, blocks = codes.shape[0], (cols + BLOCK - 1) // BLOCK
        _require(codes.is_contiguous() and scales.is_contiguous() and codes.device == scales.device, "Packed8: contiguous, on one device")
        _require(tuple(codes.shape) == (rows, blocks * BLOCK) and tuple(scales.shape) == (rows, blocks), "Packed8: whole blocks of 32 columns")
        shape = (rows, cols) if shape is None else tuple(shape)
        _require(len(shape) >= 1 and shape[-1] == cols and all(n >= 0 for n in shape) and math.prod(shape[:-1]) == rows,
                 f"Packed8: a shape of {rows} rows of {cols} columns")
        self._codes, self._scales, self._both = codes, scales, None
        self._rows, self._cols, self._ld, self._device, self._shape = rows, cols, blocks * BLOCK, codes.device, shape

    @classmethod
    def _new(cls, on, like, rows: int, cols: int, shape):
        """Codes and scales in one allocation; tensors of them are made when they are asked for."""
        p = object.__new__(cls)
        blocks = (cols + BLOCK - 1) // BLOCK
        p._codes = p._scales = None
        p._both = on.empty(like, (rows * blocks * (BLOCK + 1),), torch.int8)
        p._rows, p._cols, p._ld, p._shape, p._device = rows, cols, blocks * BLOCK, shape, on.dev
        return p

    def _pointers(self):
        if self._both is None:
            return self._codes.data_ptr(), self._scales.data_ptr()
        at = self._both.data_ptr()
        return at, at + self._rows * self._ld

    rows = property(lambda self: self._rows)
    cols = property(lambda self: self._cols)
    ld = property(lambda self: self._ld)
    shape = property(lambda self: self._shape)
    device = property(lambda self: self._device)

    @property
    def codes(self):
        if self._codes is None:
            self._codes = self._both[:self._rows * self._ld].view(self._rows, self._ld)
        return self._codes

    @property
    def scales(self):
        if self._scales is None:
            self._scales = self._both[self._rows * self._ld:].view(torch.uint8).view(self._rows, self._ld // BLOCK)
        return self._scales

    @property
    def nbytes(self) -> int:
        return self._rows * (self._ld + self._ld // BLOCK)


def _fail(what: str):
    raise rinr.RinrError(rinr.E_ARG, what)


def _no_graph(what: str):
    if torch.is_grad_enabled():
        _fail(what + ": keeps no graph for tensors that require gradients; torch.no_grad(), or a torch.autograd.Function around it and its backward operator")


def _mat(t, what: str):
    """(pointer, rows, columns, distance between rows) of a tensor's rows."""
    if t.requires_grad:
        _no_graph(what)
    shape = t.shape
    if len(shape) != 2:
        if not shape or shape[-1] < 1:
            _fail(what + ": at least one column")
        try:
            t = t.view(-1, shape[-1])
        except RuntimeError:
            raise rinr.RinrError(rinr.E_ARG, what + ": rows have to lie evenly apart (contiguous())") from None
        shape = t.shape
    rows, cols = shape
    step, one = t.stride()
    if one != 1 or step < cols or rows <= 1 or not t.is_cuda:
        if rows <= 1:
            step = cols or 1
        if (one != 1 and cols != 1) or step < cols or not t.is_cuda:
            _fail(what + ": on the GPU, columns side by side, rows apart")
    return t.data_ptr(), rows, cols, step


class _Here:
    """A call on the current GPU and stream."""
    __slots__ = ("dev", "ptr")

    def __init__(self, dev, ptr):
        self.dev, self.ptr = dev, ptr

    def empty(self, like, shape, dtype):
        return like.new_empty(shape) if like.dtype == dtype else like.new_empty(shape, dtype=dtype)

    def close(self):
        pass


class _There(_Here):
    """A call on another GPU or stream than the current one: outputs and scratch memory are of that stream, and inputs are held until it has done with them."""
    __slots__ = ("_guard", "_side", "_stream")

    def __init__(self, dev, stream):
        self._guard = self._side = self._stream = None
        if dev.index != torch.cuda.current_device():
            self._guard = torch.cuda.device(dev)
            self._guard.__enter__()
        try:
            super().__init__(dev, rinr._stream_ptr(stream))
            if stream is not None:
                s = stream if isinstance(stream, torch.cuda.Stream) else \
                    (torch.cuda.ExternalStream(self.ptr, device=dev) if self.ptr else torch.cuda.default_stream(dev))
                self._side, self._stream = torch.cuda.stream(s), s
        except BaseException:
            self.close()                                               # what is no stream leaves the caller on its GPU
            raise

    def empty(self, like, shape, dtype):
        if self._side is None:
            return torch.empty(shape, dtype=dtype, device=self.dev)
        here = torch.cuda.current_stream(self.dev)
        with self._side:
            t = torch.empty(shape, dtype=dtype, device=self.dev)
        t.record_stream(here)                                          # where the caller goes on with it
        return t

    def hold(self, *inputs):
        for t in inputs:
            if type(t) is Packed8:
                self.hold(*((t._codes, t._scales) if t._both is None else (t._both,)))
            elif t is not None:
                t.record_stream(self._stream)

    def close(self):
        if self._guard is not None:
            self._guard.__exit__(None, None, None)
            self._guard = None


# the current GPU, and a GPU's current stream, without an object for them (as in rinr._stream_ptr)
_device = getattr(torch._C, "_cuda_getDevice", None)
_current = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _on(dev, stream):
    if stream is None and _device is not None and _current is not None:
        i = dev.index
        if _device() == i:
            return _Here(dev, _current(i) or None)
    return _There(dev, stream)


def _call(fn, need, args, like, on, what):
    """A call that may need scratch memory (`need` says how much)."""
    rc = fn(args, None, 0, on.ptr)
    if rc == rinr.E_NULL:
        size = need(args)
        if size:
            work = on.empty(like, (size,), torch.uint8)
            rc = fn(args, work.data_ptr(), size, on.ptr)
    if rc:
        raise rinr.RinrError(rc, what)


def _operand(x, dtype, dt: int, what: str):
    """(pointer, rows, columns, distance, scales, type) of a tensor of `dtype` or of a Packed8."""
    if type(x) is Packed8:
        if x.device.type != "cuda":
            _fail(what + ": on the GPU")
        pc, ps = x._pointers()
        return pc, x._rows, x._cols, x._ld, ps, PACKED8
    if x.dtype != dtype:
        _fail(f"{what}: {dtype} or Packed8")
    p, rows, cols, step = _mat(x, what)
    return p, rows, cols, step, 0, dt


def _vector(v, n: int, dev, what: str):
    if v.requires_grad:
        _no_graph(what)
    if v.dtype != torch.float32 or v.shape != (n,) or not v.is_contiguous() or v.device != dev:
        _fail(f"{what}: a float32 vector of {n} on {dev}")
    return v.data_ptr()


def _act(name: str, what: str) -> int:
    k = ACTS.get(name)
    if k is None:
        _fail(f"{what}: act is one of {', '.join(ACTS)}")
    return k


def _alike(t, dtype, shape, dev, what: str):
    if t.dtype != dtype or t.shape != shape or t.device != dev:
        _fail(f"{what}: {dtype} {tuple(shape)} on {dev}")
    return _mat(t, what)


def _weights(w, what: str):
    if w.dtype not in TYPES or w.dim() != 2:
        _fail(what + ": w is a bfloat16, float16 or float32 matrix")
    m = _mat(w, what)
    if not m[1] or not m[2]:
        _fail(what + ": w has inputs and outputs")
    return m


def linear(x, w, bias=None, act: str = "none", w0: float = 30.0, residual=None, keep_z: Optional[str] = None, out=None, stream=None):
    """rinr_linear: act(x w' + bias) + residual, of w's type.  x: tensor [..., n_in] of that type or Packed8; bias: float32 [n_out].

    keep_z: "packed" or "tensor" keeps x w' + bias for the backward pass; then (y, z) is returned."""
    L, what = _lib or lib(), "rinr_linear"
    pw, n_out, n_in, ldw = _weights(w, what)
    dtype, dev = w.dtype, w.device
    px, rows, cols, ldx, psx, tx = _operand(x, dtype, TYPES[dtype], what)
    if cols != n_in or x.device != dev:
        _fail(f"{what}: x has {cols} columns on {x.device}, w takes {n_in} on {dev}")
    if keep_z not in (None, "packed", "tensor"):
        _fail(what + ': keep_z is None, "packed" or "tensor"')
    ka, dt = _act(act, what), TYPES[dtype]
    pb = 0 if bias is None else _vector(bias, n_out, dev, "rinr_linear bias")
    shape = (rows, n_out) if len(x.shape) == 2 else (*x.shape[:-1], n_out)
    pr = ldr = 0
    if residual is not None:
        pr, _, _, ldr = _alike(residual, dtype, shape, dev, "rinr_linear residual")
    if out is not None:
        py, _, _, ldy = _alike(out, dtype, shape, dev, "rinr_linear out")
    on = _on(dev, stream)
    try:
        if stream is not None:
            on.hold(x, w, bias, residual, out)
        if out is None:
            out = on.empty(w, shape, dtype)
            py, ldy = out.data_ptr(), n_out
        z, pz, ldz, psz, tz = None, 0, 0, 0, 0
        if keep_z == "packed":
            z = Packed8._new(on, w, rows, n_out, shape)
            (pz, psz), ldz, tz = z._pointers(), z._ld, PACKED8
        elif keep_z is not None:
            z = on.empty(w, shape, dtype)
            pz, ldz, tz = z.data_ptr(), n_out, dt
        a = _LINEAR.pack(rows, n_in, n_out, px, ldx, psx, pw, ldw, pb, pr, ldr, py, ldy, pz, ldz, psz, dt, tx, tz, ka, w0, 0)
        _call(L.rinr_linear, L.rinr_linear_workspace_bytes, a, w, on, what)
    finally:
        on.close()
    return out if keep_z is None else (out, z)


def linear_backward(dy, x, w, act: str = "none", w0: float = 30.0, z=None, x_act: str = "none", need_dx: bool = True, need_dw: bool = True,
                    need_db: bool = True, stream=None):
    """rinr_linear_backward: (dx, dw, dbias) of y = act(z), z = x w' + bias, each None where it is not needed.

    z: what linear kept, where act is not "none".  x_act: x is what an activation was taken of (the z that the layer before kept): the
    layer's input was x_act(x), and dx is the gradient of x itself.  The gradient of linear's residual is dy."""
    L, what = _lib or lib(), "rinr_linear_backward"
    pw, n_out, n_in, ldw = _weights(w, what)
    dtype, dev = w.dtype, w.device
    px, rows, cols, ldx, psx, tx = _operand(x, dtype, TYPES[dtype], what)
    if cols != n_in or x.device != dev:
        _fail(f"{what}: x has {cols} columns on {x.device}, w takes {n_in} on {dev}")
    pdy, _, _, lddy = _alike(dy, dtype, (*x.shape[:-1], n_out), dev, "rinr_linear_backward dy")
    ka, kx = _act(act, what), _act(x_act, what)
    if (z is not None) != (ka != 0):
        _fail(what + ": z, where there is an activation")
    pz, ldz, psz, tz = 0, 0, 0, 0
    if z is not None:
        pz, zr, zc, ldz, psz, tz = _operand(z, dtype, TYPES[dtype], what)
        if zr != rows or zc != n_out or z.device != dev:
            _fail(f"{what}: z has {zr} x {zc} on {z.device}, dy {rows} x {n_out} on {dev}")
    on = _on(dev, stream)
    try:
        if stream is not None:
            on.hold(dy, x, w, z)
        dx = on.empty(w, x.shape, dtype) if need_dx else None
        dw = on.empty(w, (n_out, n_in), dtype) if need_dw else None
        db = on.empty(w, (n_out,), torch.float32) if need_db else None
        a = _LINEAR_GRAD.pack(rows, n_in, n_out, pdy, lddy, px, ldx, psx, pw, ldw, pz, ldz, psz, 0 if dx is None else dx.data_ptr(), n_in,
                              0 if dw is None else dw.data_ptr(), n_in, 0 if db is None else db.data_ptr(), TYPES[dtype], tx, tz, ka, kx, w0)
        _call(L.rinr_linear_backward, L.rinr_linear_backward_workspace_bytes, a, w, on, what)
    finally:
        on.close()
    return dx, dw, db


def rms_norm(x, gain, eps: float = 1e-6, residual=None, packed: bool = False, stream=None):
    """rinr_rms_norm: (y, h) with h = x + residual (x itself where there is none) and y = gain h / sqrt(mean(h^2) + eps) over the last
    dimension, of x's type or, with `packed`, a Packed8."""
    L, what = _lib or lib(), "rinr_rms_norm"
    dtype, dev, shape = x.dtype, x.device, x.shape
    if dtype not in TYPES:
        _fail(what + ": bfloat16, float16 or float32")
    px, rows, cols, ldx = _mat(x, what)
    pg, dt = _vector(gain, cols, dev, "rinr_rms_norm gain"), TYPES[dtype]
    pr = ldr = 0
    if residual is not None:
        pr, _, _, ldr = _alike(residual, dtype, shape, dev, "rinr_rms_norm residual")
    on = _on(dev, stream)
    try:
        if stream is not None:
            on.hold(x, gain, residual)
        h = x if residual is None else on.empty(x, shape, dtype)
        if packed:
            y = Packed8._new(on, x, rows, cols, tuple(shape))
            (py, psy), ldy, ty = y._pointers(), y._ld, PACKED8
        else:
            y = on.empty(x, shape, dtype)
            py, ldy, psy, ty = y.data_ptr(), cols, 0, dt
        a = _NORM.pack(rows, cols, px, ldx, pr, ldr, pg, py, ldy, psy, 0 if residual is None else h.data_ptr(), cols, dt, ty, eps, 0)
        rinr._check(L.rinr_rms_norm(a, on.ptr), what)
    finally:
        on.close()
    return y, h


def rms_norm_backward(dy, h, gain, eps: float = 1e-6, dres=None, need_dgain: bool = True, stream=None):
    """rinr_rms_norm_backward: (dh, dgain).  dh is the gradient of x and of the residual alike; dres: the gradient that arrives at h on
    another path, added to it."""
    L, what = _lib or lib(), "rinr_rms_norm_backward"
    dtype, dev, shape = h.dtype, h.device, h.shape
    if dtype not in TYPES:
        _fail(what + ": bfloat16, float16 or float32")
    ph, rows, cols, ldh = _mat(h, what)
    pg = _vector(gain, cols, dev, "rinr_rms_norm_backward gain")
    pdy, _, _, lddy = _alike(dy, dtype, shape, dev, "rinr_rms_norm_backward dy")
    pd = ldd = 0
    if dres is not None:
        pd, _, _, ldd = _alike(dres, dtype, shape, dev, "rinr_rms_norm_backward dres")
    on = _on(dev, stream)
    try:
        if stream is not None:
            on.hold(dy, h, gain, dres)
        dh = on.empty(h, shape, dtype)
        dgain = on.empty(h, (cols,), torch.float32) if need_dgain else None
        need = L.rinr_rms_norm_backward_workspace_bytes(rows, cols) if need_dgain else 0
        work = on.empty(h, (need,), torch.uint8) if need else None
        a = _NORM_GRAD.pack(rows, cols, pdy, lddy, ph, ldh, pg, pd, ldd, dh.data_ptr(), cols, 0 if dgain is None else dgain.data_ptr(), TYPES[dtype], eps)
        rinr._check(L.rinr_rms_norm_backward(a, None if work is None else work.data_ptr(), need, on.ptr), what)
    finally:
        on.close()
    return dh, dgain


def pack8(x, stream=None) -> Packed8:
    """rinr_pack8: a tensor's rows in 8 bits."""
    L, what = _lib or lib(), "rinr_pack8"
    if x.dtype not in TYPES:
        _fail(what + ": bfloat16, float16 or float32")
    px, rows, cols, ldx = _mat(x, what)
    on = _on(x.device, stream)
    try:
        if stream is not None:
            on.hold(x)
        p = Packed8._new(on, x, rows, cols, tuple(x.shape))
        pc, ps = p._pointers()
        rinr._check(L.rinr_pack8(rows, cols, px, ldx, TYPES[x.dtype], pc, p.ld, ps, on.ptr), what)
    finally:
        on.close()
    return p


def unpack8(p: Packed8, dtype=torch.bfloat16, act: str = "none", w0: float = 30.0, stream=None):
    """rinr_unpack8: the values of a Packed8, or an activation of them, as a tensor of `dtype`."""
    L, what = _lib or lib(), "rinr_unpack8"
    if dtype not in TYPES or p.device.type != "cuda":
        _fail(what + ": bfloat16, float16 or float32, on the GPU")
    ka = _act(act, what)
    pc, ps = p._pointers()
    on = _on(p.device, stream)
    try:
        if stream is not None:
            on.hold(p)
        x = on.empty(p._codes if p._both is None else p._both, p.shape, dtype)
        rinr._check(L.rinr_unpack8(p.rows, p.cols, pc, p.ld, ps, ka, w0, x.data_ptr(), p.cols, TYPES[dtype], on.ptr), what)
    finally:
        on.close()
    return x

"""The operators of residual blocks (include/lf_operators.h) for torch tensors: one Python function per C entry point, same
names, that marshals arguments and returns the lf_status; and objects that keep an operator's outputs and workspace, as
`LeapfrogNet` keeps a net's.

An object's outputs are overwritten by its next pass.  Work is enqueued on torch's current stream of the object's device.
`rows` of an object is the most rows it takes: a call's inputs may have fewer, and its outputs then are views of the first ones."""
from __future__ import annotations

import ctypes as C
from typing import Optional

from .binding import LF_BF16, LF_EINVAL, LF_F32, LF_OK, LfError, lib

LF_MATRIX_F32, LF_MATRIX_BF16, LF_MATRIX_E4M3 = range(3)
LF_ACT_NONE, LF_ACT_SIGMOID, LF_ACT_RELU, LF_ACT_SILU, LF_ACT_GELU = range(5)
ACTIVATIONS = {"none": LF_ACT_NONE, "sigmoid": LF_ACT_SIGMOID, "relu": LF_ACT_RELU, "silu": LF_ACT_SILU,
               "gelu": LF_ACT_GELU}
GROUP = 32          # values of a row that share a scale in 8 bits


class lf_matrix(C.Structure):
    """lf_matrix of lf_operators.h: device pointers and row strides."""
    _fields_ = [("data", C.c_void_p), ("ld", C.c_longlong), ("scales", C.c_void_p), ("scale_ld", C.c_longlong),
                ("type", C.c_int)]


_bound = None


def _lib() -> C.CDLL:
    global _bound
    if _bound is None:
        L = lib()
        i, sz, vp, f, mp = C.c_int, C.c_size_t, C.c_void_p, C.c_float, C.POINTER(lf_matrix)
        for name, res, args in [
                ("lf_checkpoint_save", i, [i, i, mp, mp, vp]),
                ("lf_checkpoint_load", i, [i, i, mp, mp, vp]),
                ("lf_norm_forward", i, [i, i, mp, mp, vp, f, mp, mp, vp, vp]),
                ("lf_norm_workspace_bytes", sz, [i, i]),
                ("lf_norm_backward", i, [i, i, mp, mp, vp, vp, mp, mp, vp, vp, sz, vp]),
                ("lf_linear_workspace_bytes", sz, [i, i, i, i]),
                ("lf_linear_forward", i, [i, i, i, mp, mp, vp, i, mp, mp, mp, vp, sz, vp]),
                ("lf_linear_backward_workspace_bytes", sz, [i, i, i, i]),
                ("lf_linear_backward", i, [i, i, i, mp, mp, i, mp, mp, mp, mp, vp, vp, sz, vp]),
                ("lf_operator_error", C.c_char_p, [])]:
            fn = getattr(L, name)
            fn.restype, fn.argtypes = res, args
        _bound = L
    return _bound


# ---- thin functions: matrices are lf_matrix or None, vectors and streams addresses (0: NULL) --------------------------
def lf_checkpoint_save(rows, cols, x, out, hip_stream=0) -> int:
    return _lib().lf_checkpoint_save(rows, cols, x, out, hip_stream)


def lf_checkpoint_load(rows, cols, in_, out, hip_stream=0) -> int:
    return _lib().lf_checkpoint_load(rows, cols, in_, out, hip_stream)


def lf_norm_forward(rows, cols, x, branch, gain, eps, sum_, y, rstd, hip_stream=0) -> int:
    return _lib().lf_norm_forward(rows, cols, x, branch, gain, eps, sum_, y, rstd, hip_stream)


def lf_norm_workspace_bytes(rows, cols) -> int:
    return _lib().lf_norm_workspace_bytes(rows, cols)


def lf_norm_backward(rows, cols, dy, sum_, gain, rstd, dsum, dx, dgain, workspace, workspace_bytes, hip_stream=0) -> int:
    return _lib().lf_norm_backward(rows, cols, dy, sum_, gain, rstd, dsum, dx, dgain, workspace, workspace_bytes,
                                   hip_stream)


def lf_linear_workspace_bytes(rows, outputs, inputs, dt) -> int:
    return _lib().lf_linear_workspace_bytes(rows, outputs, inputs, dt)


def lf_linear_forward(rows, outputs, inputs, x, w, bias, act, residual, y, z, workspace, workspace_bytes,
                      hip_stream=0) -> int:
    return _lib().lf_linear_forward(rows, outputs, inputs, x, w, bias, act, residual, y, z, workspace, workspace_bytes,
                                    hip_stream)


def lf_linear_backward_workspace_bytes(rows, outputs, inputs, dt) -> int:
    return _lib().lf_linear_backward_workspace_bytes(rows, outputs, inputs, dt)


def lf_linear_backward(rows, outputs, inputs, dy, z, act, x, w, dx, dw, db, workspace, workspace_bytes,
                       hip_stream=0) -> int:
    return _lib().lf_linear_backward(rows, outputs, inputs, dy, z, act, x, w, dx, dw, db, workspace, workspace_bytes,
                                     hip_stream)


def lf_operator_error() -> str:
    return _lib().lf_operator_error().decode()


# ---- objects ---------------------------------------------------------------------------------------------------------
def _torch():
    import torch
    return torch


def _storage(dtype):
    """(torch type, matrix type, lf_dtype) of "f32", "bf16" or a torch type."""
    t = _torch()
    if dtype in ("f32", t.float32):
        return t.float32, LF_MATRIX_F32, LF_F32
    if dtype in ("bf16", t.bfloat16):
        return t.bfloat16, LF_MATRIX_BF16, LF_BF16
    raise LfError(LF_EINVAL, f"storage type {dtype!r}: f32 and bf16 are supported")


def _check(st: int) -> None:
    if st != LF_OK:
        raise LfError(st, lf_operator_error())


class E4M3Matrix:
    """rows x cols values in 8 bits: `codes` (uint8, [rows][cols rounded up to whole groups of 32], e4m3) and `scales`
    (uint8, one power of two per group: 2^(byte - 127))."""

    def __init__(self, rows: int, cols: int, device: str = "cuda:0"):
        t = _torch()
        groups = -(-cols // GROUP)
        self._set(t.empty((rows, groups * GROUP), dtype=t.uint8, device=device),
                  t.empty((rows, groups), dtype=t.uint8, device=device), cols)

    @classmethod
    def of(cls, codes, scales, cols: int) -> "E4M3Matrix":
        """The matrix that codes and scales (uint8 tensors of the shapes above, on one GPU) stand for.  They are
        not copied."""
        t = _torch()
        m = cls.__new__(cls)
        groups = -(-cols // GROUP)
        for name, x, width in (("codes", codes, groups * GROUP), ("scales", scales, groups)):
            if x.dtype != t.uint8 or x.dim() != 2 or x.shape[1] != width or (width > 1 and x.stride(1) != 1):
                raise LfError(LF_EINVAL, f"{name} of a matrix in 8 bits with {cols} columns: uint8 [rows][{width}] with "
                                         f"contiguous rows is needed, got {x.dtype} {list(x.shape)}")
        if codes.shape[0] != scales.shape[0] or codes.device != scales.device:
            raise LfError(LF_EINVAL, "codes and scales have different rows or devices")
        m._set(codes, scales, cols)
        return m

    def _set(self, codes, scales, cols):
        self.codes, self.scales, self.cols = codes, scales, cols
        self.rows, self.device = codes.shape[0], codes.device
        # (a stride of a matrix of one row or none says nothing)
        self._m = lf_matrix(codes.data_ptr(), max(codes.stride(0), codes.shape[1]), scales.data_ptr(),
                            max(scales.stride(0), scales.shape[1]), LF_MATRIX_E4M3)

    @property
    def shape(self):
        return (self.rows, self.cols)

    def first(self, rows: int) -> "E4M3Matrix":
        """The first rows (no copy)."""
        return self if rows == self.rows else E4M3Matrix.of(self.codes[:rows], self.scales[:rows], self.cols)

    def save(self, x) -> "E4M3Matrix":
        """Keep x ([rows][cols], f32 or bf16)."""
        _check(lf_checkpoint_save(self.rows, self.cols, _matrix("x", x, self.rows, self.cols, self.device), self._m,
                                  _stream(self.device)))
        return self

    def load(self, out=None, dtype="bf16"):
        """The values, in `out` or a new tensor of the type."""
        if out is None:
            out = _torch().empty(self.rows, self.cols, dtype=_storage(dtype)[0], device=self.device)
        _check(lf_checkpoint_load(self.rows, self.cols, self._m, _matrix("out", out, self.rows, self.cols, self.device),
                                  _stream(self.device)))
        return out


def _stream(device) -> int:
    return _torch().cuda.current_stream(device).cuda_stream


_TYPES = None


def _matrix(name, x, rows, cols, device):
    """lf_matrix of a tensor or a matrix in 8 bits, which must be rows x cols on the device; None stays None."""
    global _TYPES
    if x is None:
        return None
    if isinstance(x, E4M3Matrix):
        if x.rows != rows or x.cols != cols or x.device != device:
            raise LfError(LF_EINVAL, f"{name}: {rows} x {cols} on {device} is needed, got {x.rows} x {x.cols} on {x.device}")
        return x._m
    if _TYPES is None:
        t = _torch()
        _TYPES = {t.float32: LF_MATRIX_F32, t.bfloat16: LF_MATRIX_BF16}
    kind = _TYPES.get(x.dtype)
    if kind is None or x.shape != (rows, cols) or x.device != device:
        raise LfError(LF_EINVAL, f"{name}: {rows} x {cols}, f32 or bf16, on {device} is needed, got {list(x.shape)}, "
                                 f"{x.dtype}, on {x.device}")
    ld, inner = x.stride()
    if rows <= 1:
        ld = max(ld, cols)          # a stride of one row says nothing
    if inner != 1 and cols > 1:
        raise LfError(LF_EINVAL, f"{name}: rows have to be contiguous, strides are {x.stride()}")
    return lf_matrix(x.data_ptr(), ld, None, 0, kind)


def _vector(name, x, n, device) -> int:
    if x is None:
        return 0
    if x.dtype != _torch().float32 or x.shape != (n,) or x.device != device or (n > 1 and x.stride(0) != 1):
        raise LfError(LF_EINVAL, f"{name}: {n} contiguous f32 on {device} are needed, got {list(x.shape)}, {x.dtype}, on "
                                 f"{x.device}")
    return x.data_ptr()


class _Operator:
    """What the operators below share: device, storage type, outputs, workspace."""

    def __init__(self, rows, dtype, passes, device):
        t = _torch()
        if passes not in ("forward", "backward", "both"):
            raise LfError(LF_EINVAL, f"passes = {passes!r}: forward, backward or both")
        self.rows, self.device = rows, t.device(device)
        if self.device.index is None:
            self.device = t.device(self.device.type, 0)
        self.dtype, _, self._dt = _storage(dtype)
        self._forward, self._backward = passes != "backward", passes != "forward"

    def _new(self, name, rows, cols, kind):
        """A matrix of the storage type or, "e4m3", in 8 bits; None for "none"; a matrix of the caller's is taken as it is."""
        if isinstance(kind, (_torch().Tensor, E4M3Matrix)):
            _matrix(name, kind, rows, cols, self.device)
            return kind
        if isinstance(kind, str) and kind == "none":
            return None
        if isinstance(kind, str) and kind == "e4m3":
            return E4M3Matrix(rows, cols, self.device)
        return _torch().empty((rows, cols), dtype=_storage(kind)[0], device=self.device)

    def _scratch(self, nbytes):
        return _torch().empty(nbytes, dtype=_torch().uint8, device=self.device)

    def _need(self, have, what):
        if not have:
            raise LfError(LF_EINVAL, f"this object was made without its {what} pass")

    def _count(self, x):
        rows = x.shape[0]
        if rows > self.rows:
            raise LfError(LF_EINVAL, f"{rows} rows, the object was made for {self.rows}")
        return rows

    def _first(self, x, rows):
        if x is None or rows == self.rows:
            return x
        return x.first(rows) if isinstance(x, E4M3Matrix) else x[:rows]


class RmsNorm(_Operator):
    """Root-mean-square norm with the residual's addition:  sum = x + branch,  y = sum / rms(sum) * gain.

    gain: f32 [cols], ones at first.  out: type of y, dtype or "e4m3".  After `forward`: sum, y (a tensor or an E4M3Matrix),
    rstd.  After `backward`: dx (the gradient of x and of branch), dgain.  out, sum and dx may be matrices of the caller's to
    write to (sum: x or branch itself, too; dx: dsum itself, too); sum may be "none"."""

    def __init__(self, rows: int, cols: int, dtype="bf16", out=None, eps: float = 1e-6, passes: str = "both", sum=None,
                 dx=None, device: str = "cuda:0"):
        super().__init__(rows, dtype, passes, device)
        t = _torch()
        self.cols, self.eps = cols, eps
        f32 = dict(dtype=t.float32, device=self.device)
        self.gain = t.ones(cols, **f32)
        self._sum = self._y = self._dx = self.sum = self.y = self.dx = self.rstd = self.dgain = None
        if self._forward:
            self._sum = self._new("sum", rows, cols, self.dtype if sum is None else sum)
            self._y = self._new("out", rows, cols, self.dtype if out is None else out)
            self._rstd = t.empty(rows, **f32)
        if self._backward:
            self._dx = self._new("dx", rows, cols, self.dtype if dx is None else dx)
            self.dgain = t.empty(cols, **f32)
            self._workspace = self._scratch(lf_norm_workspace_bytes(rows, cols))

    def forward(self, x, branch=None):
        self._need(self._forward, "forward")
        n, c, dev = self._count(x), self.cols, self.device
        self.sum, self.y, self.rstd = (self._first(v, n) for v in (self._sum, self._y, self._rstd))
        _check(lf_norm_forward(n, c, _matrix("x", x, n, c, dev), _matrix("branch", branch, n, c, dev),
                               _vector("gain", self.gain, c, dev), self.eps, _matrix("sum", self.sum, n, c, dev),
                               _matrix("y", self.y, n, c, dev), self.rstd.data_ptr(), _stream(dev)))
        return self.y

    def backward(self, dy, dsum=None, stored=None, rstd=None):
        """From dy and the gradient that reaches the sum on other ways.  stored: the sum, if not the last forward pass's,
        in the storage type or in 8 bits; rstd likewise."""
        self._need(self._backward, "backward")
        n, c, dev = self._count(dy), self.cols, self.device
        stored, rstd = self.sum if stored is None else stored, self.rstd if rstd is None else rstd
        self.dx = self._first(self._dx, n)
        _check(lf_norm_backward(n, c, _matrix("dy", dy, n, c, dev), _matrix("stored", stored, n, c, dev),
                                _vector("gain", self.gain, c, dev), _vector("rstd", rstd, n, dev),
                                _matrix("dsum", dsum, n, c, dev), _matrix("dx", self.dx, n, c, dev),
                                self.dgain.data_ptr(), self._workspace.data_ptr(), self._workspace.numel(), _stream(dev)))
        return self.dx


class Linear(_Operator):
    """Matrix product with bias, activation and residual:  z = x w^T + b,  y = act(z) + residual.

    y: storage type ("f32", "bf16", None: dtype) or "e4m3"; z, what the backward pass needs of an activation:
    the same, or "none".  dw: type of the weights' gradient, dtype or "f32".  After `forward`: y, z.  After `backward`: dx, dw, db.
    y, z, dx and dw may be matrices of the caller's to write to, workspace scratch that operators on one stream share
    (uint8; `workspace_bytes` of it at least)."""

    def __init__(self, rows: int, outputs: int, inputs: int, dtype="bf16", act: str = "none", y=None, z="none", dx=None,
                 dw=None, workspace=None, passes: str = "both", device: str = "cuda:0"):
        super().__init__(rows, dtype, passes, device)
        if act not in ACTIVATIONS:
            raise LfError(LF_EINVAL, f"activation {act!r}: one of {sorted(ACTIVATIONS)}")
        t = _torch()
        self.outputs, self.inputs, self._act = outputs, inputs, ACTIVATIONS[act]
        self.w = self.b = self.y = self.z = self.dx = self.dw = self.db = None
        nbytes = 0
        if self._forward:
            self._y = self._new("y", rows, outputs, self.dtype if y is None else y)
            self._z = self._new("z", rows, outputs, z)
            nbytes = lf_linear_workspace_bytes(rows, outputs, inputs, self._dt)
        if self._backward:
            self._dx = self._new("dx", rows, inputs, self.dtype if dx is None else dx)
            self.dw = self._new("dw", outputs, inputs, self.dtype if dw is None else dw)
            self.db = t.empty(outputs, dtype=t.float32, device=self.device)
            nbytes = max(nbytes, lf_linear_backward_workspace_bytes(rows, outputs, inputs, self._dt))
        self.workspace_bytes = nbytes
        self._workspace = self._scratch(nbytes) if workspace is None else workspace

    def set_params(self, w, b=None) -> None:
        """w: [outputs][inputs] of the storage type; b: [outputs] f32 or None.  Kept by reference."""
        _matrix("w", w, self.outputs, self.inputs, self.device)
        _vector("b", b, self.outputs, self.device)
        self.w, self.b = w, b

    def forward(self, x, residual=None):
        self._need(self._forward, "forward")
        n, o, i, dev = self._count(x), self.outputs, self.inputs, self.device
        self.y, self.z = self._first(self._y, n), self._first(self._z, n)
        _check(lf_linear_forward(n, o, i, _matrix("x", x, n, i, dev), _matrix("w", self.w, o, i, dev),
                                 _vector("b", self.b, o, dev), self._act, _matrix("residual", residual, n, o, dev),
                                 _matrix("y", self.y, n, o, dev), _matrix("z", self.z, n, o, dev),
                                 self._workspace.data_ptr(), self._workspace.numel(), _stream(dev)))
        return self.y

    def backward(self, dy, x, z=None):
        """From dy, the input of the forward pass, and z if it is not the last forward pass's."""
        self._need(self._backward, "backward")
        n, o, i, dev = self._count(dy), self.outputs, self.inputs, self.device
        z = self.z if z is None else z
        self.dx = self._first(self._dx, n)
        _check(lf_linear_backward(n, o, i, _matrix("dy", dy, n, o, dev), _matrix("z", z, n, o, dev), self._act,
                                  _matrix("x", x, n, i, dev), _matrix("w", self.w, o, i, dev),
                                  _matrix("dx", self.dx, n, i, dev), _matrix("dw", self.dw, o, i, dev),
                                  self.db.data_ptr(), self._workspace.data_ptr(), self._workspace.numel(), _stream(dev)))
        return self.dx

"""The operators of residual blocks (include/lf_operators.h) for torch tensors: one Python function per C entry point, same
names, that marshals arguments and returns the lf_status; and objects that keep an operator's outputs and workspace, as
`LeapfrogNet` keeps a net's.

An object's outputs are overwritten by its next pass.  Work is enqueued on torch's current stream of the object's device, whatever
the current device is.  A matrix in 8 bits may be loaded by several threads at once; any other object serves one thread and one
stream at a time (its outputs and its workspace are the same in every pass).
`rows` of an object is the most rows it takes: a call's inputs may have fewer, and its outputs then are views of the first ones."""
from __future__ import annotations

import ctypes as C
from typing import Optional

from .binding import LF_BF16, LF_EINVAL, LF_F32, LF_OK, LfError, lib

LF_MATRIX_F32, LF_MATRIX_BF16, LF_MATRIX_E4M3, LF_MATRIX_E4M3_128, LF_MATRIX_E4M3_TILES = range(5)
LF_ACT_NONE, LF_ACT_SIGMOID, LF_ACT_RELU, LF_ACT_SILU, LF_ACT_GELU = range(5)
ACTIVATIONS = {"none": LF_ACT_NONE, "sigmoid": LF_ACT_SIGMOID, "relu": LF_ACT_RELU, "silu": LF_ACT_SILU,
               "gelu": LF_ACT_GELU}
GROUP = 32          # values of a row that share a scale in 8 bits
BLOCK = 128         # the same, in blocks of 128


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
                ("lf_layer_norm_forward", i, [i, i, mp, mp, vp, vp, f, mp, mp, vp, vp, vp]),
                ("lf_layer_norm_workspace_bytes", sz, [i, i]),
                ("lf_layer_norm_backward", i, [i, i, mp, mp, vp, vp, vp, mp, mp, vp, vp, vp, sz, vp]),
                ("lf_block_save", i, [i, i, mp, mp, mp, vp]),
                ("lf_block_load", i, [i, i, mp, mp, vp]),
                ("lf_block_linear_workspace_bytes", sz, [i, i, i]),
                ("lf_block_linear_forward", i, [i, i, i, mp, mp, vp, i, mp, mp, mp, mp, vp, sz, vp]),
                ("lf_block_linear_backward_workspace_bytes", sz, [i, i, i]),
                ("lf_block_linear_backward", i, [i, i, i, mp, mp, i, mp, mp, mp, mp, vp, vp, sz, vp]),
                ("lf_distil", i, [i, i, i, mp, mp, vp, C.c_longlong, f, vp, vp, mp, vp]),
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


def lf_layer_norm_forward(rows, cols, x, branch, gain, shift, eps, sum_, y, mean, rstd, hip_stream=0) -> int:
    return _lib().lf_layer_norm_forward(rows, cols, x, branch, gain, shift, eps, sum_, y, mean, rstd, hip_stream)


def lf_layer_norm_workspace_bytes(rows, cols) -> int:
    return _lib().lf_layer_norm_workspace_bytes(rows, cols)


def lf_layer_norm_backward(rows, cols, dy, sum_, gain, mean, rstd, dsum, dx, dgain, dshift, workspace, workspace_bytes,
                           hip_stream=0) -> int:
    return _lib().lf_layer_norm_backward(rows, cols, dy, sum_, gain, mean, rstd, dsum, dx, dgain, dshift, workspace,
                                         workspace_bytes, hip_stream)


def lf_block_save(rows, cols, x, out, out_t, hip_stream=0) -> int:
    return _lib().lf_block_save(rows, cols, x, out, out_t, hip_stream)


def lf_block_load(rows, cols, in_, out, hip_stream=0) -> int:
    return _lib().lf_block_load(rows, cols, in_, out, hip_stream)


def lf_block_linear_workspace_bytes(rows, outputs, inputs) -> int:
    return _lib().lf_block_linear_workspace_bytes(rows, outputs, inputs)


def lf_block_linear_forward(rows, outputs, inputs, x, w, bias, act, residual, y, z, x_t, workspace, workspace_bytes,
                            hip_stream=0) -> int:
    return _lib().lf_block_linear_forward(rows, outputs, inputs, x, w, bias, act, residual, y, z, x_t, workspace,
                                          workspace_bytes, hip_stream)


def lf_block_linear_backward_workspace_bytes(rows, outputs, inputs) -> int:
    return _lib().lf_block_linear_backward_workspace_bytes(rows, outputs, inputs)


def lf_block_linear_backward(rows, outputs, inputs, dy, z, act, x_t, w_t, dx, dw, db, workspace, workspace_bytes,
                             hip_stream=0) -> int:
    return _lib().lf_block_linear_backward(rows, outputs, inputs, dy, z, act, x_t, w_t, dx, dw, db, workspace,
                                           workspace_bytes, hip_stream)


def lf_distil(rows, classes, top, logits, top_logits, top_classes, top_classes_ld, temperature, weight, loss, dlogits,
              hip_stream=0) -> int:
    return _lib().lf_distil(rows, classes, top, logits, top_logits, top_classes, top_classes_ld, temperature, weight, loss,
                            dlogits, hip_stream)


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


class E4M3Matrix:
    """rows x cols values in 8 bits: `codes` (uint8, [rows][cols rounded up to whole groups of 32], e4m3) and `scales`
    (uint8, one power of two per group: 2^(byte - 127), 255 a NaN; `save` writes 10 to 247)."""

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
        self.shape, self._gpu = (self.rows, cols), codes.get_device()
        # (the stride of one row or of none says nothing)
        self._m = lf_matrix(codes.data_ptr(), max(codes.stride(0), codes.shape[1]), scales.data_ptr(),
                            max(scales.stride(0), scales.shape[1]), LF_MATRIX_E4M3)

    def first(self, rows: int) -> "E4M3Matrix":
        """The first rows (no copy)."""
        return self if rows == self.rows else E4M3Matrix.of(self.codes[:rows], self.scales[:rows], self.cols)

    def save(self, x) -> "E4M3Matrix":
        """Keep x ([rows][cols], f32 or bf16)."""
        _enqueue(self._gpu, _lib().lf_checkpoint_save, self.rows, self.cols, _matrix("x", x, self.shape, self._gpu, lf_matrix()), self._m)
        return self

    def load(self, out=None, dtype="bf16"):
        """The values, in `out` or a new tensor of the type."""
        if out is None:
            out = _torch().empty(self.shape, dtype=_storage(dtype)[0], device=self.device)
        _enqueue(self._gpu, _lib().lf_checkpoint_load, self.rows, self.cols, self._m,
                 _matrix("out", out, self.shape, self._gpu, lf_matrix()))
        return out


class E4M3Blocks:
    """rows x cols values in 8 bits with blocks of 128: `codes` (uint8, [rows][cols rounded up to whole 128], e4m3) and `scales`
    (uint8, one power of two for 128 columns of a row, or with `tiles` for 128 x 128 values; rows of whole fours).  Bytes as
    E4M3Matrix's."""

    def __init__(self, rows: int, cols: int, tiles: bool = False, device: str = "cuda:0"):
        t = _torch()
        groups = -(-cols // BLOCK)
        self._set(t.empty((rows, groups * BLOCK), dtype=t.uint8, device=device),
                  t.empty((-(-rows // BLOCK) if tiles else rows, -(-groups // 4) * 4), dtype=t.uint8, device=device), cols, tiles)

    @classmethod
    def of(cls, codes, scales, cols: int, tiles: bool = False) -> "E4M3Blocks":
        """The matrix that codes and scales (uint8 tensors of the shapes above, on one GPU) stand for.  They are
        not copied."""
        t = _torch()
        m = cls.__new__(cls)
        groups = -(-cols // BLOCK)
        for name, x, width in (("codes", codes, groups * BLOCK), ("scales", scales, -(-groups // 4) * 4)):
            if x.dtype != t.uint8 or x.dim() != 2 or x.shape[1] != width or (width > 1 and x.stride(1) != 1):
                raise LfError(LF_EINVAL, f"{name} of a matrix in blocks of 128 with {cols} columns: uint8 [rows][{width}] with "
                                         f"contiguous rows is needed, got {x.dtype} {list(x.shape)}")
        if scales.shape[0] != (-(-codes.shape[0] // BLOCK) if tiles else codes.shape[0]) or codes.device != scales.device:
            raise LfError(LF_EINVAL, "codes and scales have different rows or devices")
        m._set(codes, scales, cols, tiles)
        return m

    def _set(self, codes, scales, cols, tiles):
        self.codes, self.scales, self.cols, self.tiles = codes, scales, cols, tiles
        self.rows, self.device = codes.shape[0], codes.device
        self.shape, self._gpu = (self.rows, cols), codes.get_device()
        # (the stride of one row or of none says nothing)
        self._m = lf_matrix(codes.data_ptr(), codes.stride(0) if codes.shape[0] > 1 else max(codes.stride(0), codes.shape[1]),
                            scales.data_ptr(), scales.stride(0) if scales.shape[0] > 1 else max(scales.stride(0), scales.shape[1]),
                            LF_MATRIX_E4M3_TILES if tiles else LF_MATRIX_E4M3_128)

    def first(self, rows: int) -> "E4M3Blocks":
        """The first rows (no copy)."""
        if rows == self.rows:
            return self
        return E4M3Blocks.of(self.codes[:rows], self.scales[:-(-rows // BLOCK) if self.tiles else rows], self.cols, self.tiles)

    def first_columns(self, cols: int) -> "E4M3Blocks":
        """The first columns (no copy; the rest of the last group that they share belongs to them)."""
        if cols == self.cols:
            return self
        groups = -(-cols // BLOCK)
        return E4M3Blocks.of(self.codes[:, :groups * BLOCK], self.scales[:, :-(-groups // 4) * 4], cols, self.tiles)

    def save(self, x, transposed: Optional["E4M3Blocks"] = None) -> "E4M3Blocks":
        """Keep x ([rows][cols], f32 or bf16), and in the same pass x^T in `transposed` ([cols][rows], with tiles if this has them)."""
        _enqueue(self._gpu, _lib().lf_block_save, self.rows, self.cols, _matrix("x", x, self.shape, self._gpu, lf_matrix()), self._m,
                 _matrix("transposed", transposed, (self.cols, self.rows), self._gpu, lf_matrix()))
        return self

    def load(self, out=None, dtype="bf16"):
        """The values, in `out` or a new tensor of the type."""
        if out is None:
            out = _torch().empty(self.shape, dtype=_storage(dtype)[0], device=self.device)
        _enqueue(self._gpu, _lib().lf_block_load, self.rows, self.cols, self._m,
                 _matrix("out", out, self.shape, self._gpu, lf_matrix()))
        return out


_raw_stream = _current_gpu = None


def _enqueue(gpu: int, call, *args) -> None:
    """A C call on torch's current stream of a GPU.  The GPU is the current device meanwhile: its default stream is 0, as every
    other's is.  (`torch.cuda.current_stream` makes an object for it: a microsecond a call.)"""
    global _raw_stream, _current_gpu
    if gpu < 0:
        raise LfError(LF_EINVAL, f"{call.__name__}: the operands are on the CPU, the operators run on a GPU")
    if _raw_stream is None:
        t = _torch()
        _current_gpu = getattr(t._C, "_cuda_getDevice", None) or t.cuda.current_device
        _raw_stream = getattr(t._C, "_cuda_getCurrentRawStream", None) or (lambda i: t.cuda.current_stream(i).cuda_stream)
    if _current_gpu() == gpu:
        st = call(*args, _raw_stream(gpu))
    else:
        with _torch().cuda.device(gpu):
            st = call(*args, _raw_stream(gpu))
    if st != LF_OK:
        raise LfError(st, lf_operator_error())


_TYPES = None


def _matrix(name, x, shape, gpu, m):
    """Fills m with a tensor's address and stride, or gives that of a matrix in 8 bits: x must have the shape and lie on the
    GPU.  None stays None."""
    global _TYPES
    if x is None:
        return None
    if type(x) is E4M3Matrix or type(x) is E4M3Blocks:
        if x.shape != shape or x._gpu != gpu:
            raise LfError(LF_EINVAL, f"{name}: {shape[0]} x {shape[1]} on GPU {gpu} is needed, got {x.shape} on {x.device}")
        return x._m
    if _TYPES is None:
        t = _torch()
        _TYPES = {t.float32: LF_MATRIX_F32, t.bfloat16: LF_MATRIX_BF16}
    kind = _TYPES.get(x.dtype)
    if kind is None or x.shape != shape or x.get_device() != gpu:
        raise LfError(LF_EINVAL, f"{name}: {shape[0]} x {shape[1]}, f32 or bf16, on GPU {gpu} is needed, got "
                                 f"{list(x.shape)}, {x.dtype}, on {x.device}")
    ld, inner = x.stride()
    if inner != 1 and shape[1] > 1:
        raise LfError(LF_EINVAL, f"{name}: rows have to be contiguous, strides are {x.stride()}")
    m.data, m.ld, m.type = x.data_ptr(), ld if shape[0] > 1 else max(ld, shape[1]), kind      # (one row's stride says nothing)
    return m


def _vector(name, x, n, gpu) -> int:
    if x is None:
        return 0
    if x.dtype != _torch().float32 or x.shape != (n,) or x.get_device() != gpu or (n > 1 and x.stride(0) != 1):
        raise LfError(LF_EINVAL, f"{name}: {n} contiguous f32 on GPU {gpu} are needed, got {list(x.shape)}, {x.dtype}, on "
                                 f"{x.device}")
    return x.data_ptr()


class _Kept:
    """A vector that an object keeps by reference: checked when it is given, and again where it has moved."""

    def __init__(self, name, x, n, gpu):
        self.name, self.n, self.gpu = name, n, gpu
        self.at = _vector(name, x, n, gpu)

    def address(self, x) -> int:
        if x is None:
            return 0
        if x.data_ptr() != self.at:
            self.at = _vector(self.name, x, self.n, self.gpu)
        return self.at


class _Operator:
    """What the operators below share: device, storage type, outputs, workspace."""

    def __init__(self, rows, dtype, passes, device):
        t = _torch()
        if passes not in ("forward", "backward", "both"):
            raise LfError(LF_EINVAL, f"passes = {passes!r}: forward, backward or both")
        self.rows, self.device = rows, t.device(device)
        if self.device.type == "cuda" and self.device.index is None:
            self.device = t.device("cuda", t.cuda.current_device())
        self._gpu = -1 if self.device.type == "cpu" else self.device.index
        self.dtype, _, self._dt = _storage(dtype)
        self._forward, self._backward = passes != "backward", passes != "forward"
        self._in = [lf_matrix() for _ in range(4)]          # of a call's inputs
        self._whole = {}                                   # lf_matrix of an output of all rows

    def _new(self, name, rows, cols, kind):
        """An output: a matrix of the storage type or in 8 bits ("e4m3", and "e4m3_128" in blocks of 128); None for "none"; a matrix of
        the caller's is taken as it is."""
        if isinstance(kind, str) and kind == "none":
            return None
        if isinstance(kind, str) and kind == "e4m3":
            kind = E4M3Matrix(rows, cols, self.device)
        elif isinstance(kind, str) and kind == "e4m3_128":
            kind = E4M3Blocks(rows, cols, device=self.device)
        elif not isinstance(kind, (_torch().Tensor, E4M3Matrix, E4M3Blocks)):
            kind = _torch().empty((rows, cols), dtype=_storage(kind)[0], device=self.device)
        self._whole[name] = _matrix(name, kind, (rows, cols), self._gpu, lf_matrix())
        return kind

    def _some(self, name, whole, n):
        """(the first n rows of an output, their lf_matrix)"""
        if n == self.rows or whole is None:
            return whole, self._whole.get(name)
        part = whole.first(n) if isinstance(whole, (E4M3Matrix, E4M3Blocks)) else whole[:n]
        return part, _matrix(name, part, (n, whole.shape[1]), self._gpu, lf_matrix())

    def _scratch(self, nbytes):
        return _torch().empty(nbytes, dtype=_torch().uint8, device=self.device)

    def _begin(self, x, have, what):
        """Rows of a call's input."""
        n = x.shape[0]
        if n > self.rows:
            raise LfError(LF_EINVAL, f"{n} rows, the object was made for {self.rows}")
        if not have:
            raise LfError(LF_EINVAL, f"this object was made without its {what} pass")
        return n


class RmsNorm(_Operator):
    """Root-mean-square norm with the residual's addition:  sum = x + branch,  y = sum / rms(sum) * gain.

    gain: f32 [cols], ones at first.  out: type of y, dtype or "e4m3".  After `forward`: sum, y (a tensor or an E4M3Matrix),
    rstd.  After `backward`: dx (the gradient of x and of branch), dgain.  out, sum and dx may be matrices of the caller's to
    write to, which stay where they are (sum: x or branch itself, too; dx: dsum itself, too); sum may be "none"."""

    def __init__(self, rows: int, cols: int, dtype="bf16", out=None, eps: float = 1e-6, passes: str = "both", sum=None,
                 dx=None, device: str = "cuda:0"):
        super().__init__(rows, dtype, passes, device)
        t = _torch()
        self.cols, self.eps = cols, eps
        f32 = dict(dtype=t.float32, device=self.device)
        self.gain = t.ones(cols, **f32)          # (checked when it is set, not in every pass)
        self._sum = self._y = self._dx = self.sum = self.y = self.dx = self.rstd = self.dgain = None
        if self._forward:
            self._sum = self._new("sum", rows, cols, self.dtype if sum is None else sum)
            self._y = self._new("out", rows, cols, self.dtype if out is None else out)
            self._rstd = t.empty(rows, **f32)
        if self._backward:
            self._dx = self._new("dx", rows, cols, self.dtype if dx is None else dx)
            self.dgain = t.empty(cols, **f32)
            self.workspace_bytes = lf_norm_workspace_bytes(rows, cols)
            self._workspace = self._scratch(self.workspace_bytes)

    @property
    def gain(self):
        return self._gain

    @gain.setter
    def gain(self, gain):
        self._gain, self._kept_gain = gain, _Kept("gain", gain, self.cols, self._gpu)

    def forward(self, x, branch=None):
        n, c, gpu, m = self._begin(x, self._forward, "forward"), self.cols, self._gpu, self._in
        self.sum, msum = self._some("sum", self._sum, n)
        self.y, my = self._some("out", self._y, n)
        self.rstd = self._rstd if n == self.rows else self._rstd[:n]
        shape = (n, c)
        _enqueue(gpu, _lib().lf_norm_forward, n, c, _matrix("x", x, shape, gpu, m[0]), _matrix("branch", branch, shape, gpu, m[1]),
                 self._kept_gain.address(self._gain), self.eps, msum, my, self._rstd.data_ptr())
        return self.y

    def backward(self, dy, dsum=None, stored=None, rstd=None):
        """From dy and the gradient that reaches the sum on other ways.  stored: the sum, if not the last forward pass's,
        in the storage type or in 8 bits; rstd likewise."""
        n, c, gpu, m = self._begin(dy, self._backward, "backward"), self.cols, self._gpu, self._in
        stored, rstd = self.sum if stored is None else stored, self.rstd if rstd is None else rstd
        self.dx, mdx = self._some("dx", self._dx, n)
        shape = (n, c)
        _enqueue(gpu, _lib().lf_norm_backward, n, c, _matrix("dy", dy, shape, gpu, m[0]), _matrix("stored", stored, shape, gpu, m[1]),
                 self._kept_gain.address(self._gain), _vector("rstd", rstd, n, gpu), _matrix("dsum", dsum, shape, gpu, m[2]), mdx,
                 self.dgain.data_ptr(), self._workspace.data_ptr(), self.workspace_bytes)
        return self.dx


class LayerNorm(_Operator):
    """Layer norm with the residual's addition:  sum = x + branch,  y = (sum - mean) / deviation * gain + shift.

    gain, shift: f32 [cols], ones and zeros at first.  out: type of y, dtype, "e4m3" or "e4m3_128".  After `forward`: sum, y (a tensor,
    an E4M3Matrix or an E4M3Blocks), mean, rstd.  After `backward`: dx (the gradient of x and of branch), dgain, dshift.  out, sum and
    dx may be matrices of the caller's, as RmsNorm's."""

    def __init__(self, rows: int, cols: int, dtype="bf16", out=None, eps: float = 1e-5, passes: str = "both", sum=None,
                 dx=None, device: str = "cuda:0"):
        super().__init__(rows, dtype, passes, device)
        t = _torch()
        self.cols, self.eps = cols, eps
        f32 = dict(dtype=t.float32, device=self.device)
        self.gain, self.shift = t.ones(cols, **f32), t.zeros(cols, **f32)
        self._sum = self._y = self._dx = self.sum = self.y = self.dx = self.mean = self.rstd = self.dgain = self.dshift = None
        if self._forward:
            self._sum = self._new("sum", rows, cols, self.dtype if sum is None else sum)
            self._y = self._new("out", rows, cols, self.dtype if out is None else out)
            self._mean, self._rstd = t.empty(rows, **f32), t.empty(rows, **f32)
        if self._backward:
            self._dx = self._new("dx", rows, cols, self.dtype if dx is None else dx)
            self.dgain, self.dshift = t.empty(cols, **f32), t.empty(cols, **f32)
            self.workspace_bytes = lf_layer_norm_workspace_bytes(rows, cols)
            self._workspace = self._scratch(self.workspace_bytes)

    @property
    def gain(self):
        return self._gain

    @gain.setter
    def gain(self, gain):
        self._gain, self._kept_gain = gain, _Kept("gain", gain, self.cols, self._gpu)

    @property
    def shift(self):
        return self._shift

    @shift.setter
    def shift(self, shift):
        self._shift, self._kept_shift = shift, _Kept("shift", shift, self.cols, self._gpu)

    def forward(self, x, branch=None):
        n, c, gpu, m = self._begin(x, self._forward, "forward"), self.cols, self._gpu, self._in
        self.sum, msum = self._some("sum", self._sum, n)
        self.y, my = self._some("out", self._y, n)
        whole = n == self.rows
        self.mean, self.rstd = self._mean if whole else self._mean[:n], self._rstd if whole else self._rstd[:n]
        shape = (n, c)
        _enqueue(gpu, _lib().lf_layer_norm_forward, n, c, _matrix("x", x, shape, gpu, m[0]), _matrix("branch", branch, shape, gpu, m[1]),
                 self._kept_gain.address(self._gain), self._kept_shift.address(self._shift), self.eps, msum, my,
                 self._mean.data_ptr(), self._rstd.data_ptr())
        return self.y

    def backward(self, dy, dsum=None, stored=None, mean=None, rstd=None):
        """From dy and the gradient that reaches the sum on other ways.  stored: the sum, if not the last forward pass's,
        in the storage type or in an E4M3Matrix; mean and rstd likewise."""
        n, c, gpu, m = self._begin(dy, self._backward, "backward"), self.cols, self._gpu, self._in
        stored = self.sum if stored is None else stored
        mean, rstd = self.mean if mean is None else mean, self.rstd if rstd is None else rstd
        self.dx, mdx = self._some("dx", self._dx, n)
        shape = (n, c)
        _enqueue(gpu, _lib().lf_layer_norm_backward, n, c, _matrix("dy", dy, shape, gpu, m[0]), _matrix("stored", stored, shape, gpu, m[1]),
                 self._kept_gain.address(self._gain), _vector("mean", mean, n, gpu), _vector("rstd", rstd, n, gpu),
                 _matrix("dsum", dsum, shape, gpu, m[2]), mdx, self.dgain.data_ptr(), self.dshift.data_ptr(),
                 self._workspace.data_ptr(), self.workspace_bytes)
        return self.dx


class Linear(_Operator):
    """Matrix product with bias, activation and residual:  z = x w^T + b,  y = act(z) + residual.

    y: storage type ("f32", "bf16", None: dtype) or "e4m3"; z, what the backward pass needs of an activation:
    the same, or "none".  dw: type of the weights' gradient, dtype or "f32".  After `forward`: y, z.  After `backward`: dx, dw, db.
    y, z, dx and dw may be matrices of the caller's to write to, which stay where they are, workspace scratch that operators on one stream share
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
        if workspace is not None and (workspace.dtype != t.uint8 or workspace.get_device() != self._gpu
                                      or not workspace.is_contiguous() or workspace.numel() < nbytes):
            raise LfError(LF_EINVAL, f"workspace: {nbytes} contiguous uint8 on GPU {self._gpu} are needed")
        self._workspace = self._scratch(nbytes) if workspace is None else workspace

    def set_params(self, w, b=None) -> None:
        """Register w ([outputs][inputs], storage type) and b ([outputs] f32, or None).  They are kept by reference: the
        data may change between passes, and where it lies."""
        kept = _Kept("b", b, self.outputs, self._gpu)
        self._look_at(w)
        self.w, self.b, self._kept_b = w, b, kept

    def _look_at(self, w):
        if w.dtype != self.dtype:
            raise LfError(LF_EINVAL, f"w: {self.dtype} is needed, got {w.dtype}")
        self._mw = _matrix("w", w, (self.outputs, self.inputs), self._gpu, lf_matrix())
        self._seen = w.data_ptr(), w.stride(), w.shape

    def _weights(self):
        w = self.w
        if w is None:
            raise LfError(LF_EINVAL, "w is NULL: set_params gives the weights")
        if (w.data_ptr(), w.stride(), w.shape) != self._seen or w.dtype != self.dtype:
            self._look_at(w)
        return self._mw

    def forward(self, x, residual=None):
        n, o, i, gpu, m = self._begin(x, self._forward, "forward"), self.outputs, self.inputs, self._gpu, self._in
        self.y, my = self._some("y", self._y, n)
        self.z, mz = self._some("z", self._z, n)
        _enqueue(gpu, _lib().lf_linear_forward, n, o, i, _matrix("x", x, (n, i), gpu, m[0]), self._weights(), self._kept_b.address(self.b),
                 self._act, _matrix("residual", residual, (n, o), gpu, m[1]), my, mz, self._workspace.data_ptr(),
                 self.workspace_bytes)
        return self.y

    def backward(self, dy, x, z=None):
        """From dy, the input of the forward pass, and z if it is not the last forward pass's.  Without an activation z is not
        looked at."""
        n, o, i, gpu, m = self._begin(dy, self._backward, "backward"), self.outputs, self.inputs, self._gpu, self._in
        z = None if self._act == LF_ACT_NONE else self.z if z is None else z
        self.dx, mdx = self._some("dx", self._dx, n)
        _enqueue(gpu, _lib().lf_linear_backward, n, o, i, _matrix("dy", dy, (n, o), gpu, m[0]),
                 _matrix("z", z, (n, o), gpu, m[1]), self._act, _matrix("x", x, (n, i), gpu, m[2]),
                 self._weights(), mdx, self._whole["dw"], self.db.data_ptr(), self._workspace.data_ptr(), self.workspace_bytes)
        return self.dx


class BlockLinear(_Operator):
    """Matrix product with bias, activation and residual of operands in 8 bits with blocks of 128:  z = x w^T + b,  y = act(z) + residual.

    `set_params` keeps the weights in 8 bits (w8, and w8_t for the backward pass), `refresh` does so again after they have changed.
    x is put into 8 bits in the pass; with passes="both" its transposed codes are kept for the backward pass (x_t), an eighth
    to a quarter of what x took.  x that is an E4M3Blocks already is taken as it is, and x_t is the caller's then.  y: storage type or
    "e4m3_128"; z, what the backward pass needs of an activation: the same, or "none"; dw: dtype or "f32".  After `forward`: y, z, x_t.
    After `backward`: dx, dw, db.  y, z, dx, dw and workspace may be the caller's, as Linear's."""

    def __init__(self, rows: int, outputs: int, inputs: int, dtype="bf16", act: str = "none", y=None, z="none", dx=None,
                 dw=None, workspace=None, passes: str = "both", device: str = "cuda:0"):
        super().__init__(rows, dtype, passes, device)
        if act not in ACTIVATIONS:
            raise LfError(LF_EINVAL, f"activation {act!r}: one of {sorted(ACTIVATIONS)}")
        t = _torch()
        self.outputs, self.inputs, self._act = outputs, inputs, ACTIVATIONS[act]
        self.w = self.b = self.w8 = self.w8_t = self.y = self.z = self.dx = self.dw = self.db = self.x_t = self._x_t = None
        nbytes = 0
        if self._forward:
            self._y = self._new("y", rows, outputs, self.dtype if y is None else y)
            self._z = self._new("z", rows, outputs, z)
            nbytes = lf_block_linear_workspace_bytes(rows, outputs, inputs)
            if self._backward:
                self._x_t = E4M3Blocks(inputs, rows, device=self.device)
        if self._backward:
            self._dx = self._new("dx", rows, inputs, self.dtype if dx is None else dx)
            self.dw = self._new("dw", outputs, inputs, self.dtype if dw is None else dw)
            self.db = t.empty(outputs, dtype=t.float32, device=self.device)
            nbytes = max(nbytes, lf_block_linear_backward_workspace_bytes(rows, outputs, inputs))
        self.workspace_bytes = nbytes
        if workspace is not None and (workspace.dtype != t.uint8 or workspace.get_device() != self._gpu
                                      or not workspace.is_contiguous() or workspace.numel() < nbytes):
            raise LfError(LF_EINVAL, f"workspace: {nbytes} contiguous uint8 on GPU {self._gpu} are needed")
        self._workspace = self._scratch(nbytes) if workspace is None else workspace

    def set_params(self, w, b=None, w_t=None) -> None:
        """Register w ([outputs][inputs], f32 or bf16) and b ([outputs] f32, or None), and keep w in 8 bits.  w and b are kept by reference:
        after w has changed, `refresh`.  w may be in 8 bits already, an E4M3Blocks with tiles; the backward pass needs w_t then, its
        transposed."""
        self._register(w, b, w_t)
        self.refresh()

    def _register(self, w, b=None, w_t=None) -> None:
        kept = _Kept("b", b, self.outputs, self._gpu)
        shape, gpu = (self.outputs, self.inputs), self._gpu
        if isinstance(w, E4M3Blocks):
            _matrix("w", w, shape, gpu, lf_matrix())
            if self._backward and not isinstance(w_t, E4M3Blocks):
                raise LfError(LF_EINVAL, "w_t: the backward pass takes weights in 8 bits transposed")
            _matrix("w_t", w_t, shape[::-1], gpu, lf_matrix())
            self.w, self.w8, self.w8_t = None, w, w_t if self._backward else None
        else:
            _matrix("w", w, shape, gpu, lf_matrix())
            if w_t is not None:
                raise LfError(LF_EINVAL, "w_t goes with weights in 8 bits")
            # (matrices of the caller's, of an earlier call, are left as they are)
            if self.w is None:
                self.w8 = E4M3Blocks(*shape, tiles=True, device=self.device) if self._forward else None
                self.w8_t = E4M3Blocks(*shape[::-1], tiles=True, device=self.device) if self._backward else None
            self.w = w
        self.b, self._kept_b = b, kept

    def refresh(self) -> None:
        """Keep the weights as they are now in 8 bits.  (Weights that were given in 8 bits are read as they lie.)"""
        if self.w is None:
            if self.w8 is None and self.w8_t is None:
                raise LfError(LF_EINVAL, "w is NULL: set_params gives the weights")
            return
        _enqueue(self._gpu, _lib().lf_block_save, self.outputs, self.inputs,
                 _matrix("w", self.w, (self.outputs, self.inputs), self._gpu, lf_matrix()), self.w8 and self.w8._m, self.w8_t and self.w8_t._m)

    def _weights(self, w8):
        if w8 is None:
            raise LfError(LF_EINVAL, "w is NULL: set_params gives the weights")
        return w8._m

    def forward(self, x, residual=None):
        n, o, i, gpu, m = self._begin(x, self._forward, "forward"), self.outputs, self.inputs, self._gpu, self._in
        self.y, my = self._some("y", self._y, n)
        self.z, mz = self._some("z", self._z, n)
        self.x_t = None if self._x_t is None or isinstance(x, E4M3Blocks) else self._x_t.first_columns(n)
        _enqueue(gpu, _lib().lf_block_linear_forward, n, o, i, _matrix("x", x, (n, i), gpu, m[0]), self._weights(self.w8),
                 self._kept_b.address(self.b), self._act, _matrix("residual", residual, (n, o), gpu, m[1]), my, mz,
                 None if self.x_t is None else self.x_t._m, self._workspace.data_ptr(), self.workspace_bytes)
        return self.y

    def backward(self, dy, x_t=None, z=None):
        """From dy, the transposed input of the forward pass (E4M3Blocks, [inputs][rows]) and z, if they are not the last forward pass's.
        Without an activation z is not looked at."""
        n, o, i, gpu, m = self._begin(dy, self._backward, "backward"), self.outputs, self.inputs, self._gpu, self._in
        x_t = self.x_t if x_t is None else x_t
        z = None if self._act == LF_ACT_NONE else self.z if z is None else z
        self.dx, mdx = self._some("dx", self._dx, n)
        _enqueue(gpu, _lib().lf_block_linear_backward, n, o, i, _matrix("dy", dy, (n, o), gpu, m[0]), _matrix("z", z, (n, o), gpu, m[1]),
                 self._act, _matrix("x_t", x_t, (i, n), gpu, m[2]), self._weights(self.w8_t), mdx, self._whole["dw"], self.db.data_ptr(),
                 self._workspace.data_ptr(), self.workspace_bytes)
        return self.dx


class Distillation(_Operator):
    """Distillation loss of each row from a teacher's top logits:  p = softmax(t / T) over the row's `top` entries,
    q = softmax(logits / T) over the classes,  loss = weight T^2 sum p (log p - log q),  and its gradient in the same pass.

    passes: "both", or "forward" for the loss alone.  After `forward`: loss (f32), dlogits (the gradient of the rows' losses, their
    weights in it).  dlogits may be a matrix of the caller's to write to, the logits of the call themselves among them."""

    def __init__(self, rows: int, classes: int, top: int, dtype="bf16", temperature: float = 1.0, passes: str = "both", dlogits=None,
                 device: str = "cuda:0"):
        super().__init__(rows, dtype, passes, device)
        if not self._forward:
            raise LfError(LF_EINVAL, f"passes = {passes!r}: forward or both (the gradient is the loss's pass's)")
        self.classes, self.top, self.temperature = classes, top, temperature
        self.loss = self.dlogits = self._dlogits = None
        self._loss = _torch().empty(rows, dtype=_torch().float32, device=self.device)
        if self._backward:
            self._dlogits = self._new("dlogits", rows, classes, self.dtype if dlogits is None else dlogits)

    def forward(self, logits, top_logits, top_classes, weight=None):
        """top_logits: [rows][top], f32 or bf16; top_classes: [rows][top] int32, negative where there is no entry; weight: [rows] f32, None
        for ones."""
        n, gpu, m = self._begin(logits, True, "forward"), self._gpu, self._in
        shape = (n, self.top)
        if (top_classes.dtype != _torch().int32 or top_classes.shape != shape or top_classes.get_device() != gpu
                or (self.top > 1 and top_classes.stride(1) != 1)):
            raise LfError(LF_EINVAL, f"top_classes: {n} x {self.top} int32 with contiguous rows on GPU {gpu} are needed, got "
                                     f"{list(top_classes.shape)}, {top_classes.dtype}, on {top_classes.device}")
        self.loss = self._loss if n == self.rows else self._loss[:n]
        self.dlogits, mdl = self._some("dlogits", self._dlogits, n)
        _enqueue(gpu, _lib().lf_distil, n, self.classes, self.top, _matrix("logits", logits, (n, self.classes), gpu, m[0]),
                 _matrix("top_logits", top_logits, shape, gpu, m[1]), top_classes.data_ptr(),
                 top_classes.stride(0) if n > 1 else max(top_classes.stride(0), self.top), self.temperature,
                 _vector("weight", weight, n, gpu), self._loss.data_ptr(), mdl)
        return self.loss

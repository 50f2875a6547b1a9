"""The layers of the computation graphs as operators on device tensors.

Residual add + layer norm, matrix products grouped by ragged row ranges, and
the softmax loss, each with its backward pass: hand-written gfx950 kernels in
``libpase.so`` behind the C ABI of ``include/pase_operators.h``, which says
what each computes.  The functions here check their arguments, allocate the
outputs and enqueue the work on the current stream of the tensors' device;
nothing waits for it.  A refused argument raises `PaseError`.

``layer_norm``, ``grouped_matmul`` and ``softmax_loss`` are differentiable, once
(`torch.autograd`; a second derivative raises); the others are the passes they are made of.
"""
from __future__ import annotations

import ctypes as C
import functools
import inspect

import torch
from torch.autograd.function import once_differentiable

from . import pase
from .pase import INVALID_ARGUMENT, PaseError

BF16, FP16, FP32 = range(3)
_DTYPES = {torch.bfloat16: BF16, torch.float16: FP16, torch.float32: FP32}
NORM_MAX_WIDTH = 16384
MAX_GROUPS = 65536

EXPORTS = ["pase_operator_error", "pase_layer_norm_forward", "pase_layer_norm_workspace",
           "pase_layer_norm_backward", "pase_grouped_matmul_forward", "pase_grouped_matmul_workspace",
           "pase_grouped_matmul_backward", "pase_softmax_loss_forward", "pase_softmax_loss_forward_parts",
           "pase_softmax_loss_grad", "pase_softmax_loss_backward", "pase_softmax_loss_backward_parts"]

_lib = None


def load():
    """libpase.so with the operators' signatures set."""
    global _lib
    if _lib is not None:
        return _lib
    L = pase.load()
    P, I, U32, U64, I64, F = C.c_void_p, C.c_int, C.c_uint32, C.c_uint64, C.c_int64, C.c_float
    sig = {
        "pase_layer_norm_forward": [I, I, U64, U64, P, U64, P, U64, P, P, F, P, U64, P, U64, P, P, P],
        "pase_layer_norm_workspace": [I, U64, U64, P],
        "pase_layer_norm_backward": [I, I, U64, U64, P, U64, P, U64, P, U64, P, P, P, P, U64, P, P, P, U64, P],
        "pase_grouped_matmul_forward": [I, I, U64, U32, U64, U64, P, U64, P, P, I, P, U64, P],
        "pase_grouped_matmul_workspace": [I, I, U64, U32, U64, U64, P],
        "pase_grouped_matmul_backward": [I, I, U64, U32, U64, U64, P, U64, P, U64, P, P, I, P, U64, P, P, U64, P],
        "pase_softmax_loss_forward": [I, U64, U64, P, U64, P, I, I64, P, P, P],
        "pase_softmax_loss_forward_parts": [I, U64, U64, P, U64, P, I, I64, P, P, P, P],
        "pase_softmax_loss_grad": [I, U64, U64, P, U64, P, I, I64, P, U64, P, P, P, U64, P],
        "pase_softmax_loss_backward": [I, U64, U64, P, U64, P, I, I64, P, P, U64, P, U64, P],
        "pase_softmax_loss_backward_parts": [I, U64, U64, P, U64, P, I, I64, P, P, P, U64, P, U64, P],
    }
    for name, args in sig.items():
        f = getattr(L, name)
        f.restype, f.argtypes = C.c_int, args
    L.pase_operator_error.restype, L.pase_operator_error.argtypes = C.c_char_p, []
    _lib = L
    return L


def _refuse(msg: str):
    raise PaseError(INVALID_ARGUMENT, msg)


def _check(rc: int):
    if rc:
        raise PaseError(rc, load().pase_operator_error().decode())


_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (
    lambda index: torch.cuda.current_stream(index).cuda_stream)


def _on_device(name):
    """Runs an operator with the device of its argument `name` as the
    current one; the operator enqueues on that device's current stream."""
    def wrap(fn):
        which = list(inspect.signature(fn).parameters).index(name)

        @functools.wraps(fn)
        def run(*args, **kw):
            t = args[which] if len(args) > which else kw.get(name)
            if t is None:
                return fn(*args, **kw)   # says which argument is missing
            index = t.get_device()
            if index < 0 or index == torch.cuda.current_device():   # a host tensor is refused by the checks
                return fn(*args, **kw)
            with torch.cuda.device(index):
                return fn(*args, **kw)
        return run
    return wrap


def _matrix(name, t, like=None, rows=None, cols=None):
    """Checks a [rows, cols] argument, of the type and device of `like`, and gives its row stride."""
    if t.dim() != 2:
        _refuse(f"{name} has {t.dim()} dimensions, 2 are wanted")
    have_rows, have_cols = t.shape
    if like is not None:
        if have_rows != rows or have_cols != cols:
            _refuse(f"{name} is {tuple(t.shape)}, ({rows}, {cols}) is wanted")
        _same(name, t, like.dtype, like)
    elif t.get_device() < 0:
        _refuse(f"{name} is not on a GPU")
    ld, step = t.stride()
    if step != 1 and have_cols > 1:
        _refuse(f"the elements of a row of {name} are {step} apart, not adjacent")
    if have_rows < 2:
        return have_cols   # whatever the distance to a next row is, also beyond the operators' limit
    if ld < have_cols:
        _refuse(f"the rows of {name} overlap")
    return ld


def _same(name, t, dtype, like):
    if dtype is not None and t.dtype is not dtype:
        _refuse(f"{name} is {t.dtype}, {dtype} is wanted")
    if t.get_device() != like.get_device():
        _refuse(f"{name} is on {t.device}, not on {like.device}")


def _vector(name, t, n, dtype, like):
    if t.dim() != 1 or t.shape[0] != n:
        _refuse(f"{name} is {tuple(t.shape)}, ({n},) is wanted")
    _same(name, t, dtype, like)
    if n > 1 and t.stride(0) != 1:
        _refuse(f"{name} is not contiguous")
    return t.data_ptr()


def _dtype(name, dtype):
    d = _DTYPES.get(dtype)
    if d is None:
        _refuse(f"{name} is {dtype}: bfloat16, float16 or float32 is wanted")
    return d


def _index(name, t, n, like):
    """Checks a vector of n int32 or int64 and gives (pointer, is 64 bits)."""
    wide = t.dtype is torch.int64
    if not wide and t.dtype is not torch.int32:
        _refuse(f"{name} is {t.dtype}: int32 or int64 is wanted")
    return _vector(name, t, n, None, like), 1 if wide else 0


@functools.lru_cache(maxsize=4096)
def _bytes(name, *sizes):
    """Workspace that the library asks for at these types and sizes."""
    need = C.c_uint64()
    _check(getattr(load(), name)(*sizes, C.byref(need)))
    return need.value


def _workspace(like, name, *sizes):
    """A workspace for one call: (tensor, pointer, bytes)."""
    need = _bytes(name, *sizes)
    if not need:
        return None, None, 0
    ws = like.new_empty(need, dtype=torch.uint8)
    return ws, ws.data_ptr(), need


# ------------------------------------------------------------------ layer norm
def _params(gain, bias, width, x):
    if gain.dtype is not x.dtype and gain.dtype is not torch.float32:
        _refuse(f"gain is {gain.dtype}: {x.dtype} or torch.float32 is wanted")
    g = _vector("gain", gain, width, None, x)
    return g, _vector("bias", bias, width, gain.dtype, x) if bias is not None else None


@_on_device("x")
def layer_norm_forward(x, gain, bias=None, residual=None, eps: float = 1e-5):
    """(y, z, mean, rstd) of the rows of z = x + residual [rows, width]; without
    a residual z is x itself.  gain, bias: [width], in x's type or float32."""
    d = _dtype("x", x.dtype)
    ldx = _matrix("x", x)
    rows, width = x.shape
    g, b = _params(gain, bias, width, x)
    y = x.new_empty((rows, width))
    mean, rstd = x.new_empty((2, rows), dtype=torch.float32).unbind()
    z, r, ldr, zp = x, None, 0, None
    if residual is not None:
        ldr, r = _matrix("residual", residual, x, rows, width), residual.data_ptr()
        z = x.new_empty((rows, width))
        zp = z.data_ptr()
    _check(load().pase_layer_norm_forward(
        d, _DTYPES[gain.dtype], rows, width, x.data_ptr(), ldx, r, ldr, g, b, eps, y.data_ptr(), width, zp, width,
        mean.data_ptr(), rstd.data_ptr(), _raw_stream(x.get_device())))
    return y, z, mean, rstd


@_on_device("dy")
def layer_norm_backward(dy, z, gain, mean, rstd, dz=None):
    """(dx, dgain, dbias): dx is the gradient of x and of the residual alike.
    dz: the gradient that reaches z other than through the norm."""
    d = _dtype("dy", dy.dtype)
    lddy = _matrix("dy", dy)
    rows, width = dy.shape
    ldz = _matrix("z", z, dy, rows, width)
    lddz = _matrix("dz", dz, dy, rows, width) if dz is not None else 0
    g, _ = _params(gain, None, width, dy)
    m = _vector("mean", mean, rows, torch.float32, dy)
    r = _vector("rstd", rstd, rows, torch.float32, dy)
    L = load()
    ws, wp, have = _workspace(dy, "pase_layer_norm_workspace", d, rows, width)
    dx = dy.new_empty((rows, width))
    dgain, dbias = dy.new_empty((2, width), dtype=gain.dtype).unbind()
    _check(L.pase_layer_norm_backward(
        d, _DTYPES[gain.dtype], rows, width, dy.data_ptr(), lddy, z.data_ptr(), ldz,
        dz.data_ptr() if dz is not None else None, lddz, g, m, r, dx.data_ptr(), width, dgain.data_ptr(),
        dbias.data_ptr(), wp, have, _raw_stream(dy.get_device())))
    return dx, dgain, dbias


# ------------------------------------------------------------------ grouped products
def _groups(w, like):
    if w.dim() != 3:
        _refuse(f"w has {w.dim()} dimensions, (groups, n, k) is wanted")
    _same("w", w, like.dtype, like)
    if not w.is_contiguous():
        _refuse("w is not contiguous")
    return w.shape


def _out_dtype(name, want, dtype):
    want = want or dtype
    if want is not dtype and want is not torch.float32:
        _refuse(f"{name} is {want}: {dtype} or torch.float32 is wanted")
    return want


@_on_device("x")
def grouped_matmul_forward(x, w, offsets, out_dtype=None):
    """y[t] = w[e] x[t] for the rows t of each group e, offsets[e] .. offsets[e + 1] - 1.

    x: [rows, k]; w: [groups, n, k], contiguous; offsets: [groups + 1], int32 or
    int64, on the device.  Rows of no group get 0.  The result is [rows, n] in
    x's type, or float32 on request."""
    d = _dtype("x", x.dtype)
    ldx = _matrix("x", x)
    groups, n, k = _groups(w, x)
    rows, width = x.shape
    if width != k:
        _refuse(f"x has rows of {width}, w of {k}")
    off, off64 = _index("offsets", offsets, groups + 1, x)
    out = _out_dtype("out_dtype", out_dtype, x.dtype)
    y = x.new_empty((rows, n), dtype=out)
    _check(load().pase_grouped_matmul_forward(d, _DTYPES[out], rows, groups, n, k, x.data_ptr(), ldx, w.data_ptr(), off,
                                              off64, y.data_ptr(), n, _raw_stream(x.get_device())))
    return y


@_on_device("dy")
def grouped_matmul_backward(dy, x, w, offsets, grad_dtype=None, need_dx: bool = True, need_dw: bool = True):
    """(dx, dw) of `grouped_matmul_forward`: dx in dy's type, dw [groups, n, k] in
    dy's type or float32 (grad_dtype).  One that is not needed is None."""
    d = _dtype("dy", dy.dtype)
    lddy = _matrix("dy", dy)
    groups, n, k = _groups(w, dy)
    rows, width = dy.shape
    if width != n:
        _refuse(f"dy has rows of {width}, w gives rows of {n}")
    ldx = _matrix("x", x, dy, rows, k)
    off, off64 = _index("offsets", offsets, groups + 1, dy)
    grad = _out_dtype("grad_dtype", grad_dtype, dy.dtype)
    L = load()
    dx = dy.new_empty((rows, k)) if need_dx else None
    dw, ws, wp, have = None, None, None, 0
    if need_dw:
        dw = dy.new_empty((groups, n, k), dtype=grad)
        ws, wp, have = _workspace(dy, "pase_grouped_matmul_workspace", d, _DTYPES[grad], rows, groups, n, k)
    _check(L.pase_grouped_matmul_backward(
        d, _DTYPES[grad], rows, groups, n, k, dy.data_ptr(), lddy, x.data_ptr(), ldx, w.data_ptr(), off, off64,
        dx.data_ptr() if need_dx else None, k, dw.data_ptr() if need_dw else None, wp, have,
        _raw_stream(dy.get_device())))
    return dx, dw


# ------------------------------------------------------------------ softmax loss
def _loss_args(logits, targets):
    d = _dtype("logits", logits.dtype)
    ldl = _matrix("logits", logits)
    rows, classes = logits.shape
    t, t64 = _index("targets", targets, rows, logits)
    return d, ldl, rows, classes, t, t64


def _row_gradient(dloss, rows, like):
    """Pointer and stride of dloss: one a row, or one for all (a 0-d tensor, or expanded)."""
    _same("dloss", dloss, torch.float32, like)
    if dloss.dim() == 0:
        return dloss.data_ptr(), 0
    if dloss.dim() != 1 or dloss.shape[0] != rows:
        _refuse(f"dloss is {tuple(dloss.shape)}, ({rows},) or () is wanted")
    step = dloss.stride(0)
    if rows > 1 and step not in (0, 1):
        _refuse("dloss is neither contiguous nor one value for all rows")
    return dloss.data_ptr(), step if rows > 1 else 0


def _gradient_out(logits, out):
    if out is None:
        return logits.new_empty(logits.shape), logits.shape[1]
    return out, _matrix("out", out, logits, *logits.shape)


def _written(out):
    """Tells autograd that a caller's tensor was written, as an in-place torch
    operation does: what had saved it for its backward pass raises there."""
    if out is not None and not out.is_inference():   # an inference tensor has no version
        torch.autograd.graph.increment_version(out)


@_on_device("logits")
def softmax_loss_forward(logits, targets, ignore_index: int = -100, low: bool = False):
    """(loss, lse) per row of logits [rows, classes], float32.  targets: [rows],
    int32 or int64; a row whose target is ignore_index has loss 0.  With `low` also
    what the rounding of lse left of it, for a gradient without that rounding."""
    d, ldl, rows, classes, t, t64 = _loss_args(logits, targets)
    if low:
        loss, lse, rest = logits.new_empty((3, rows), dtype=torch.float32).unbind()
        _check(load().pase_softmax_loss_forward_parts(d, rows, classes, logits.data_ptr(), ldl, t, t64, ignore_index,
                                                      loss.data_ptr(), lse.data_ptr(), rest.data_ptr(),
                                                      _raw_stream(logits.get_device())))
        return loss, lse, rest
    loss, lse = logits.new_empty((2, rows), dtype=torch.float32).unbind()
    _check(load().pase_softmax_loss_forward(d, rows, classes, logits.data_ptr(), ldl, t, t64, ignore_index,
                                            loss.data_ptr(), lse.data_ptr(), _raw_stream(logits.get_device())))
    return loss, lse


@_on_device("logits")
def softmax_loss_grad(logits, targets, dloss, ignore_index: int = -100, out=None):
    """(loss, lse, dlogits) in one pass over the logits, for a gradient of the
    rows' losses that is known beforehand (dloss: float32 [rows], or one value
    for all), as where the loss is their mean.  out may be logits."""
    d, ldl, rows, classes, t, t64 = _loss_args(logits, targets)
    g, step = _row_gradient(dloss, rows, logits)
    loss, lse = logits.new_empty((2, rows), dtype=torch.float32).unbind()
    dlogits, lddl = _gradient_out(logits, out)
    _check(load().pase_softmax_loss_grad(d, rows, classes, logits.data_ptr(), ldl, t, t64, ignore_index, g, step,
                                         loss.data_ptr(), lse.data_ptr(), dlogits.data_ptr(), lddl,
                                         _raw_stream(logits.get_device())))
    _written(out)
    return loss, lse, dlogits


@_on_device("logits")
def softmax_loss_backward(dloss, logits, targets, lse, ignore_index: int = -100, out=None, lse_low=None):
    """dlogits from the lse of `softmax_loss_forward`, and what its rounding left where
    given.  out may be logits."""
    d, ldl, rows, classes, t, t64 = _loss_args(logits, targets)
    g, step = _row_gradient(dloss, rows, logits)
    s = _vector("lse", lse, rows, torch.float32, logits)
    dlogits, lddl = _gradient_out(logits, out)
    L, stream = load(), _raw_stream(logits.get_device())
    if lse_low is None:
        _check(L.pase_softmax_loss_backward(d, rows, classes, logits.data_ptr(), ldl, t, t64, ignore_index, s, g, step,
                                            dlogits.data_ptr(), lddl, stream))
    else:
        r = _vector("lse_low", lse_low, rows, torch.float32, logits)
        _check(L.pase_softmax_loss_backward_parts(d, rows, classes, logits.data_ptr(), ldl, t, t64, ignore_index, s, r, g,
                                                  step, dlogits.data_ptr(), lddl, stream))
    _written(out)
    return dlogits


# ------------------------------------------------------------------ differentiable forms
def _rows_adjacent(t):
    """t, or a copy of it when its rows are not what the operators read (a
    gradient that autograd expanded or transposed)."""
    return t if t.stride(-1) == 1 and (t.shape[0] < 2 or t.stride(0) >= t.shape[1]) else t.contiguous()


class _LayerNorm(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, gain, bias, residual, eps):
        y, z, mean, rstd = layer_norm_forward(x, gain, bias, residual, eps)
        ctx.save_for_backward(z, gain, mean, rstd)
        ctx.has = bias is not None, residual is not None
        ctx.set_materialize_grads(False)
        if residual is None:
            return y, None
        return y, z

    @staticmethod
    @once_differentiable
    def backward(ctx, dy, dz):
        z, gain, mean, rstd = ctx.saved_tensors
        bias, residual = ctx.has
        if dy is None:
            return dz, None, None, dz if residual else None, None
        dx, dgain, dbias = layer_norm_backward(_rows_adjacent(dy), z, gain, mean, rstd,
                                               _rows_adjacent(dz) if dz is not None else None)
        return dx, dgain, dbias if bias else None, dx if residual else None, None


def layer_norm(x, gain, bias=None, residual=None, eps: float = 1e-5):
    """Layer norm of x, or (y, z) of z = x + residual, both differentiable."""
    y, z = _LayerNorm.apply(x, gain, bias, residual, eps)
    return y if residual is None else (y, z)


class _GroupedMatmul(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, w, offsets):
        ctx.save_for_backward(x, w, offsets)
        return grouped_matmul_forward(x, w, offsets)

    @staticmethod
    @once_differentiable
    def backward(ctx, dy):
        x, w, offsets = ctx.saved_tensors
        dx, dw = grouped_matmul_backward(_rows_adjacent(dy), x, w, offsets, need_dx=ctx.needs_input_grad[0],
                                         need_dw=ctx.needs_input_grad[1])
        return dx, dw, None


def grouped_matmul(x, w, offsets):
    """`grouped_matmul_forward`, differentiable in x and w."""
    return _GroupedMatmul.apply(x, w, offsets)


class _SoftmaxLoss(torch.autograd.Function):
    @staticmethod
    def forward(ctx, logits, targets, ignore_index):
        loss, lse, low = softmax_loss_forward(logits, targets, ignore_index, low=True)
        ctx.save_for_backward(logits, targets, lse, low)
        ctx.ignore_index = ignore_index
        return loss

    @staticmethod
    @once_differentiable
    def backward(ctx, dloss):
        logits, targets, lse, low = ctx.saved_tensors
        if dloss.dim() == 1 and dloss.stride(0) not in (0, 1):
            dloss = dloss.contiguous()
        return softmax_loss_backward(dloss, logits, targets, lse, ctx.ignore_index, lse_low=low), None, None


def softmax_loss(logits, targets, ignore_index: int = -100):
    """The rows' losses, differentiable in the logits."""
    return _SoftmaxLoss.apply(logits, targets, ignore_index)

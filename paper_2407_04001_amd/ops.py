"""The layers of the computation graphs as operators on device tensors.

Residual add + layer norm, matrix products grouped by ragged row ranges, and
the softmax loss, each with its backward pass: hand-written gfx950 kernels in
``libpase.so`` behind the C ABI of ``include/pase_operators.h``, which says
what each computes.  The functions here check their arguments, allocate the
outputs and enqueue the work on the current stream of the tensors' device;
nothing waits for it.  A refused argument raises `PaseError`.

``layer_norm``, ``grouped_matmul`` and ``softmax_loss`` are differentiable
(`torch.autograd`); the others are the passes they are made of.
"""
from __future__ import annotations

import ctypes as C

import torch

from . import pase
from .pase import INVALID_ARGUMENT, PaseError

BF16, FP16, FP32 = range(3)
_DTYPES = {torch.bfloat16: BF16, torch.float16: FP16, torch.float32: FP32}
NORM_MAX_WIDTH = 16384
MAX_GROUPS = 65536

EXPORTS = ["pase_operator_error", "pase_layer_norm_forward", "pase_layer_norm_workspace",
           "pase_layer_norm_backward", "pase_grouped_matmul_forward", "pase_grouped_matmul_workspace",
           "pase_grouped_matmul_backward", "pase_softmax_loss_workspace", "pase_softmax_loss_forward",
           "pase_softmax_loss_grad", "pase_softmax_loss_backward"]

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
        "pase_softmax_loss_workspace": [I, U64, U64, P],
        "pase_softmax_loss_forward": [I, U64, U64, P, U64, P, I, I64, P, P, P, U64, P],
        "pase_softmax_loss_grad": [I, U64, U64, P, U64, P, I, I64, P, U64, P, P, P, U64, P, U64, P],
        "pase_softmax_loss_backward": [I, U64, U64, P, U64, P, I, I64, P, P, U64, P, U64, P],
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


class _On:
    """The device of the tensors as the current one, and its current stream."""

    __slots__ = ("stream", "guard")

    def __init__(self, device):
        self.guard = None
        if device.index != torch.cuda.current_device():
            self.guard = torch.cuda.device(device)

    def __enter__(self):
        if self.guard is not None:
            self.guard.__enter__()
        self.stream = torch.cuda.current_stream().cuda_stream
        return self.stream

    def __exit__(self, *exc):
        if self.guard is not None:
            self.guard.__exit__(*exc)


def _matrix(name, t, rows=None, cols=None, dtype=None, device=None):
    """Checks a [rows, cols] argument and gives its row stride."""
    if t.dim() != 2:
        _refuse(f"{name} has {t.dim()} dimensions, 2 are wanted")
    shape = t.shape
    if (rows is not None and shape[0] != rows) or (cols is not None and shape[1] != cols):
        _refuse(f"{name} is {tuple(shape)}, ({rows}, {cols}) is wanted")
    _device(name, t, dtype, device)
    ld, step = t.stride()
    if shape[1] > 1 and step != 1:
        _refuse(f"the elements of a row of {name} are {step} apart, not adjacent")
    if shape[0] > 1:
        if ld < shape[1]:
            _refuse(f"the rows of {name} overlap")
        return ld
    return max(ld, shape[1])


def _vector(name, t, n, dtype=None, device=None):
    if t.dim() != 1 or t.shape[0] != n:
        _refuse(f"{name} is {tuple(t.shape)}, ({n},) is wanted")
    _device(name, t, dtype, device)
    if n > 1 and t.stride(0) != 1:
        _refuse(f"{name} is not contiguous")
    return t.data_ptr()


def _device(name, t, dtype, device):
    if dtype is not None and t.dtype is not dtype:
        _refuse(f"{name} is {t.dtype}, {dtype} is wanted")
    if device is None:
        if not t.is_cuda:
            _refuse(f"{name} is not on a GPU")
    elif t.device != device:
        _refuse(f"{name} is on {t.device}, not on {device}")


def _dtype(name, dtype):
    d = _DTYPES.get(dtype)
    if d is None:
        _refuse(f"{name} is {dtype}: bfloat16, float16 or float32 is wanted")
    return d


def _index(name, t, n, device):
    """Checks a vector of n int32 or int64 and gives (pointer, is 64 bits)."""
    if t.dtype is not torch.int64 and t.dtype is not torch.int32:
        _refuse(f"{name} is {t.dtype}: int32 or int64 is wanted")
    return _vector(name, t, n, None, device), 1 if t.dtype is torch.int64 else 0


def _workspace(need: int, device):
    if not need:
        return None, 0
    return torch.empty(need, dtype=torch.uint8, device=device), need


# ------------------------------------------------------------------ layer norm
def _params(gain, bias, width, x):
    if gain.dtype is not x.dtype and gain.dtype is not torch.float32:
        _refuse(f"gain is {gain.dtype}: {x.dtype} or torch.float32 is wanted")
    g = _vector("gain", gain, width, None, x.device)
    return g, _vector("bias", bias, width, gain.dtype, x.device) if bias is not None else None


def layer_norm_forward(x, gain, bias=None, residual=None, eps: float = 1e-5):
    """(y, z, mean, rstd) of the rows of z = x + residual [rows, width]; without
    a residual z is x itself.  gain, bias: [width], in x's type or float32."""
    d = _dtype("x", x.dtype)
    ldx = _matrix("x", x)
    rows, width = x.shape
    ldr = _matrix("residual", residual, rows, width, x.dtype, x.device) if residual is not None else 0
    g, b = _params(gain, bias, width, x)
    with _On(x.device) as stream:
        y = torch.empty(rows, width, dtype=x.dtype, device=x.device)
        z = torch.empty_like(y) if residual is not None else x
        stats = torch.empty(2, rows, dtype=torch.float32, device=x.device)
        mean, rstd = stats[0], stats[1]
        _check(load().pase_layer_norm_forward(
            d, _DTYPES[gain.dtype], rows, width, x.data_ptr(), ldx,
            residual.data_ptr() if residual is not None else None, ldr, g, b, eps, y.data_ptr(), width,
            z.data_ptr() if residual is not None else None, width, mean.data_ptr(), rstd.data_ptr(), stream))
    return y, z, mean, rstd


def layer_norm_backward(dy, z, gain, mean, rstd, dz=None):
    """(dx, dgain, dbias): dx is the gradient of x and of the residual alike.
    dz: the gradient that reaches z other than through the norm."""
    d = _dtype("dy", dy.dtype)
    lddy = _matrix("dy", dy)
    rows, width = dy.shape
    device = dy.device
    ldz = _matrix("z", z, rows, width, dy.dtype, device)
    lddz = _matrix("dz", dz, rows, width, dy.dtype, device) if dz is not None else 0
    g, _ = _params(gain, None, width, dy)
    m = _vector("mean", mean, rows, torch.float32, device)
    r = _vector("rstd", rstd, rows, torch.float32, device)
    L = load()
    with _On(device) as stream:
        need = C.c_uint64()
        _check(L.pase_layer_norm_workspace(d, rows, width, C.byref(need)))
        ws, have = _workspace(need.value, device)
        dx = torch.empty(rows, width, dtype=dy.dtype, device=device)
        dparams = torch.empty(2, width, dtype=gain.dtype, device=device)
        dgain, dbias = dparams[0], dparams[1]
        _check(L.pase_layer_norm_backward(
            d, _DTYPES[gain.dtype], rows, width, dy.data_ptr(), lddy, z.data_ptr(), ldz,
            dz.data_ptr() if dz is not None else None, lddz, g, m, r, dx.data_ptr(), width, dgain.data_ptr(),
            dbias.data_ptr(), ws.data_ptr() if ws is not None else None, have, stream))
    return dx, dgain, dbias


# ------------------------------------------------------------------ grouped products
def _groups(w, offsets, dtype, device):
    if w.dim() != 3:
        _refuse(f"w has {w.dim()} dimensions, (groups, n, k) is wanted")
    _device("w", w, dtype, device)
    if not w.is_contiguous():
        _refuse("w is not contiguous")
    return w.shape


def _out_dtype(name, want, dtype):
    want = want or dtype
    if want is not dtype and want is not torch.float32:
        _refuse(f"{name} is {want}: {dtype} or torch.float32 is wanted")
    return want


def grouped_matmul_forward(x, w, offsets, out_dtype=None):
    """y[t] = w[e] x[t] for the rows t of each group e, offsets[e] .. offsets[e + 1] - 1.

    x: [rows, k]; w: [groups, n, k], contiguous; offsets: [groups + 1], int32 or
    int64, on the device.  Rows of no group get 0.  The result is [rows, n] in
    x's type, or float32 on request."""
    d = _dtype("x", x.dtype)
    ldx = _matrix("x", x)
    device = x.device
    groups, n, k = _groups(w, offsets, x.dtype, device)
    rows = x.shape[0]
    if x.shape[1] != k:
        _refuse(f"x has rows of {x.shape[1]}, w of {k}")
    off, off64 = _index("offsets", offsets, groups + 1, device)
    out = _out_dtype("out_dtype", out_dtype, x.dtype)
    with _On(device) as stream:
        y = torch.empty(rows, n, dtype=out, device=device)
        _check(load().pase_grouped_matmul_forward(d, _DTYPES[out], rows, groups, n, k, x.data_ptr(), ldx,
                                                  w.data_ptr(), off, off64, y.data_ptr(), n, stream))
    return y


def grouped_matmul_backward(dy, x, w, offsets, grad_dtype=None, need_dx: bool = True, need_dw: bool = True):
    """(dx, dw) of `grouped_matmul_forward`: dx in dy's type, dw [groups, n, k] in
    dy's type or float32 (grad_dtype).  One that is not needed is None."""
    d = _dtype("dy", dy.dtype)
    lddy = _matrix("dy", dy)
    device = dy.device
    groups, n, k = _groups(w, offsets, dy.dtype, device)
    rows = dy.shape[0]
    if dy.shape[1] != n:
        _refuse(f"dy has rows of {dy.shape[1]}, w gives rows of {n}")
    ldx = _matrix("x", x, rows, k, dy.dtype, device)
    off, off64 = _index("offsets", offsets, groups + 1, device)
    grad = _out_dtype("grad_dtype", grad_dtype, dy.dtype)
    L = load()
    with _On(device) as stream:
        dx = torch.empty(rows, k, dtype=dy.dtype, device=device) if need_dx else None
        dw = ws = None
        need = C.c_uint64()
        if need_dw:
            dw = torch.empty(groups, n, k, dtype=grad, device=device)
            _check(L.pase_grouped_matmul_workspace(d, _DTYPES[grad], rows, groups, n, k, C.byref(need)))
            ws, _ = _workspace(need.value, device)
        _check(L.pase_grouped_matmul_backward(
            d, _DTYPES[grad], rows, groups, n, k, dy.data_ptr(), lddy, x.data_ptr(), ldx, w.data_ptr(), off, off64,
            dx.data_ptr() if need_dx else None, k, dw.data_ptr() if need_dw else None,
            ws.data_ptr() if ws is not None else None, need.value, stream))
    return dx, dw


# ------------------------------------------------------------------ softmax loss
def _loss_args(logits, targets):
    d = _dtype("logits", logits.dtype)
    ldl = _matrix("logits", logits)
    rows, classes = logits.shape
    t, t64 = _index("targets", targets, rows, logits.device)
    return d, ldl, rows, classes, t, t64


def _row_gradient(dloss, rows, device):
    """Pointer and stride of dloss: one a row, or one for all (a 0-d tensor, or expanded)."""
    _device("dloss", dloss, torch.float32, device)
    if dloss.dim() == 0:
        return dloss.data_ptr(), 0
    if dloss.dim() != 1 or dloss.shape[0] != rows:
        _refuse(f"dloss is {tuple(dloss.shape)}, ({rows},) or () is wanted")
    step = dloss.stride(0)
    if rows > 1 and step not in (0, 1):
        _refuse("dloss is neither contiguous nor one value for all rows")
    return dloss.data_ptr(), step if rows > 1 else 0


def _loss(logits, targets, ignore_index, dloss, out):
    d, ldl, rows, classes, t, t64 = _loss_args(logits, targets)
    device = logits.device
    L = load()
    with _On(device) as stream:
        need = C.c_uint64()
        _check(L.pase_softmax_loss_workspace(d, rows, classes, C.byref(need)))
        ws, have = _workspace(need.value, device)
        wp = ws.data_ptr() if ws is not None else None
        both = torch.empty(2, rows, dtype=torch.float32, device=device)
        loss, lse = both[0], both[1]
        if dloss is None:
            _check(L.pase_softmax_loss_forward(d, rows, classes, logits.data_ptr(), ldl, t, t64, ignore_index,
                                               loss.data_ptr(), lse.data_ptr(), wp, have, stream))
            return loss, lse
        g, step = _row_gradient(dloss, rows, device)
        dlogits, lddl = _gradient_out(logits, out)
        _check(L.pase_softmax_loss_grad(d, rows, classes, logits.data_ptr(), ldl, t, t64, ignore_index, g, step,
                                        loss.data_ptr(), lse.data_ptr(), dlogits.data_ptr(), lddl, wp, have, stream))
        return loss, lse, dlogits


def _gradient_out(logits, out):
    if out is None:
        out = torch.empty(logits.shape, dtype=logits.dtype, device=logits.device)
        return out, logits.shape[1]
    return out, _matrix("out", out, *logits.shape, logits.dtype, logits.device)


def softmax_loss_forward(logits, targets, ignore_index: int = -100):
    """(loss, lse) per row of logits [rows, classes], float32.  targets: [rows],
    int32 or int64; a row whose target is ignore_index has loss 0."""
    return _loss(logits, targets, ignore_index, None, None)


def softmax_loss_grad(logits, targets, dloss, ignore_index: int = -100, out=None):
    """(loss, lse, dlogits) in one pass over the logits, for a gradient of the
    rows' losses that is known beforehand (dloss: float32 [rows], or one value
    for all), as where the loss is their mean.  out may be logits."""
    return _loss(logits, targets, ignore_index, dloss, out)


def softmax_loss_backward(dloss, logits, targets, lse, ignore_index: int = -100, out=None):
    """dlogits from the lse of `softmax_loss_forward`.  out may be logits."""
    d, ldl, rows, classes, t, t64 = _loss_args(logits, targets)
    device = logits.device
    g, step = _row_gradient(dloss, rows, device)
    s = _vector("lse", lse, rows, torch.float32, device)
    with _On(device) as stream:
        dlogits, lddl = _gradient_out(logits, out)
        _check(load().pase_softmax_loss_backward(d, rows, classes, logits.data_ptr(), ldl, t, t64, ignore_index, s, g,
                                                 step, dlogits.data_ptr(), lddl, stream))
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
        loss, lse = softmax_loss_forward(logits, targets, ignore_index)
        ctx.save_for_backward(logits, targets, lse)
        ctx.ignore_index = ignore_index
        return loss

    @staticmethod
    def backward(ctx, dloss):
        logits, targets, lse = ctx.saved_tensors
        if dloss.dim() == 1 and dloss.stride(0) not in (0, 1):
            dloss = dloss.contiguous()
        return softmax_loss_backward(dloss, logits, targets, lse, ctx.ignore_index), None, None


def softmax_loss(logits, targets, ignore_index: int = -100):
    """The rows' losses, differentiable in the logits."""
    return _SoftmaxLoss.apply(logits, targets, ignore_index)

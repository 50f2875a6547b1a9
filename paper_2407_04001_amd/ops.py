"""The layers of the computation graphs as operators on device tensors.

Residual add + layer norm, matrix products grouped by ragged row ranges,
attention over ragged sequences, rotary positions, dropout with the residual's
addition, and the softmax loss, each with its backward pass: hand-written gfx950 kernels in
``libpase.so`` behind the C ABI of ``include/pase_operators.h``, which says
what each computes.  The functions here check their arguments, allocate the
outputs and enqueue the work on the current stream of the tensors' device;
nothing waits for it.  A refused argument raises `PaseError`.

``layer_norm``, ``grouped_matmul``, ``attention``, ``rotary``, ``dropout`` and ``softmax_loss`` are differentiable, once
(`torch.autograd`; a second derivative raises); the others are the passes they are made of.
A HIP graph captures the passes as they are; their differentiable forms only while no eager graph of the same leaves
lives, since torch adds up a leaf's gradient on the stream of the first graph that holds it.
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
ATTENTION_MAX_DIM = 128
MAX_ROW_STRIDE = 1 << 22   # elements, of the products', attention's and the rotation's arguments

EXPORTS = ["pase_operator_error", "pase_layer_norm_forward", "pase_layer_norm_workspace",
           "pase_layer_norm_backward", "pase_grouped_matmul_forward", "pase_grouped_matmul_workspace",
           "pase_grouped_matmul_backward", "pase_softmax_loss_forward", "pase_softmax_loss_forward_parts",
           "pase_softmax_loss_grad", "pase_softmax_loss_backward", "pase_softmax_loss_backward_parts",
           "pase_attention_forward", "pase_attention_workspace", "pase_attention_backward", "pase_rotary", "pase_dropout"]

_lib = None


def load():
    """libpase.so with the operators' signatures set."""
    global _lib
    if _lib is not None:
        return _lib
    L = pase.load()
    P, I, U32, U64, I64, F = C.c_void_p, C.c_int, C.c_uint32, C.c_uint64, C.c_int64, C.c_float
    heads = [P, U64, U64]   # an argument [rows, heads, dim]
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
        "pase_attention_forward": [I, U64, U64, U32, U32, U32, U32, *heads * 3, P, P, P, I, I, F, *heads, P, P, U64, P],
        "pase_attention_workspace": [I, U64, U64, U32, U32, U32, U32, I, P],
        "pase_attention_backward": [I, U64, U64, U32, U32, U32, U32, *heads * 5, P, P, P, P, I, I, F, *heads * 3, P, U64, P],
        "pase_rotary": [I, U64, U32, U32, U32, I, I, *heads, P, I, P, F, *heads, P],
        "pase_dropout": [I, U64, U64, P, U64, P, U64, C.c_double, P, P, U64, P],
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
    if t.shape != (n,):
        _refuse(f"{name} is {tuple(t.shape)}, ({n},) is wanted")
    _same(name, t, dtype, like)
    if not t.is_contiguous():
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


# ------------------------------------------------------------------ attention
def _heads(name, t, like=None, rows=None, heads=None, dim=None):
    """Checks a [rows, heads, dim] argument and gives its pointer, row stride and head stride."""
    if t.dim() != 3:
        _refuse(f"{name} has {t.dim()} dimensions, (rows, heads, dim) is wanted")
    have_rows, have_heads, have_dim = t.shape
    if like is not None:
        if have_dim != dim or (rows is not None and have_rows != rows) or (heads is not None and have_heads != heads):
            _refuse(f"{name} is {tuple(t.shape)}, ({'...' if rows is None else rows}, {'...' if heads is None else heads}, {dim}) is wanted")
        _same(name, t, like.dtype, like)
    elif t.get_device() < 0:
        _refuse(f"{name} is not on a GPU")
    ld, hs, step = t.stride()
    if step != 1 and have_dim > 1:
        _refuse(f"the elements of a head of {name} are {step} apart, not adjacent")
    # the distance to a next row or head that is not there does not matter
    if have_heads < 2:
        hs = have_dim
    if have_rows < 2:
        ld = have_dim
    if ld < 0 or hs < 0:
        _refuse(f"{name} has negative strides")
    return t.data_ptr(), ld, hs


def _sequences(q_offsets, k_offsets, k_lengths, like):
    if q_offsets.dim() != 1 or q_offsets.shape[0] < 2:
        _refuse(f"q_offsets is {tuple(q_offsets.shape)}, (sequences + 1,) is wanted")
    n = q_offsets.shape[0] - 1
    qo, wide = _index("q_offsets", q_offsets, n + 1, like)
    ko, wide_k = _index("k_offsets", k_offsets, n + 1, like)
    kl, wide_l = _index("k_lengths", k_lengths, n, like) if k_lengths is not None else (None, wide)
    if wide != wide_k or wide != wide_l:
        _refuse("q_offsets, k_offsets and k_lengths are of different types")
    return n, qo, ko, kl, wide


def _attention_args(q, k, v, scale):
    """(dtype, rows, key rows, heads, kv heads, dim, scale) and the three arguments' pointers and strides."""
    d = _dtype("q", q.dtype)
    hq = _heads("q", q)
    rows, heads, dim = q.shape
    hk = _heads("k", k, q, dim=dim)
    key_rows, kv_heads, _ = k.shape
    hv = _heads("v", v, q, key_rows, kv_heads, dim)
    return (d, rows, key_rows), (heads, kv_heads, dim), max(dim, 1) ** -0.5 if scale is None else scale, (*hq, *hk, *hv)


@_on_device("q")
def attention_forward(q, k, v, q_offsets, k_offsets, k_lengths=None, causal: bool = False, scale=None):
    """(out, lse) of attention over ragged sequences: sequence b has the queries
    q_offsets[b] .. q_offsets[b + 1] - 1 and the keys from k_offsets[b] on, up to k_offsets[b + 1] - 1 or
    k_lengths[b] of them.  Causal: query i of n sees the keys up to i + (keys - n), so
    that the last one sees all, as where new tokens follow kept ones.

    q: [rows, heads, dim]; k, v: [key rows, kv heads, dim], each read by heads / kv heads heads next to each
    other; rows and heads any distance apart that keeps them from overlapping (rows up to 2 ** 22).  Offsets and lengths: int32 or int64,
    alike, on the device.  scale: dim ** -0.5 unless given.  out: [rows, heads, dim];
    lse: float32 [heads, rows].  Queries that see no key, and rows of no sequence, have out 0
    and lse -inf."""
    (d, rows, key_rows), (heads, kv_heads, dim), scale, args = _attention_args(q, k, v, scale)
    n, qo, ko, kl, wide = _sequences(q_offsets, k_offsets, k_lengths, q)
    L = load()
    ws, wp, have = _workspace(q, "pase_attention_workspace", d, rows, key_rows, n, heads, kv_heads, dim, 0)
    out = q.new_empty(rows, heads, dim)
    lse = q.new_empty(heads, rows, dtype=torch.float32)
    _check(L.pase_attention_forward(d, rows, key_rows, n, heads, kv_heads, dim, *args, qo, ko, kl, wide, bool(causal), scale,
                                    out.data_ptr(), heads * dim, dim, lse.data_ptr(), wp, have, _raw_stream(q.get_device())))
    return out, lse


@_on_device("dout")
def attention_backward(dout, q, k, v, out, lse, q_offsets, k_offsets, k_lengths=None, causal: bool = False, scale=None):
    """(dq, dk, dv) from the out and lse of `attention_forward`: dk and dv summed over
    the heads that share them, 0 for keys that no sequence has."""
    (d, rows, key_rows), (heads, kv_heads, dim), scale, args = _attention_args(q, k, v, scale)
    hdo = _heads("dout", dout, q, rows, heads, dim)
    ho = _heads("out", out, q, rows, heads, dim)
    if lse.shape != (heads, rows) or not lse.is_contiguous():
        _refuse(f"lse is {tuple(lse.shape)}, contiguous ({heads}, {rows}) is wanted")
    _same("lse", lse, torch.float32, q)
    n, qo, ko, kl, wide = _sequences(q_offsets, k_offsets, k_lengths, q)
    L = load()
    ws, wp, have = _workspace(q, "pase_attention_workspace", d, rows, key_rows, n, heads, kv_heads, dim, 1)
    dq = q.new_empty(rows, heads, dim)
    dk, dv = q.new_empty(key_rows, kv_heads, dim), q.new_empty(key_rows, kv_heads, dim)
    _check(L.pase_attention_backward(d, rows, key_rows, n, heads, kv_heads, dim, *hdo, *args, *ho, lse.data_ptr(), qo, ko, kl,
                                     wide, bool(causal), scale, dq.data_ptr(), heads * dim, dim, dk.data_ptr(),
                                     kv_heads * dim, dim, dv.data_ptr(), kv_heads * dim, dim, wp, have,
                                     _raw_stream(q.get_device())))
    return dq, dk, dv


# ------------------------------------------------------------------ rotary positions
def rotary_frequencies(turned: int, base: float = 10000.0, factor: float = 1.0, trained=None, slow: float = 1.0,
                       fast: float = 32.0, device="cuda"):
    """Frequencies of the turned / 2 pairs for `rotary`, float64: base ** (-2 i / turned), divided by
    `factor` for sequences that many times as long.  With `trained`, the length trained on, by
    parts (Peng, Quesnelle, Fan, Shippole 2023): pairs that turn more than `fast` times over that length keep their
    frequency, those below `slow` turns are divided, those between are mixed in proportion to their turns."""
    if turned < 2 or turned % 2:
        _refuse(f"{turned} elements cannot be turned in pairs")
    if not factor > 0 or not base > 0 or (trained is not None and not 0 < slow < fast):
        _refuse("base and factor are positive, and slow is below fast")
    f = base ** (-torch.arange(0, turned, 2, dtype=torch.float64, device=device) / turned)
    if trained is None:
        return f / factor
    kept = ((trained * f / 6.283185307179586 - slow) / (fast - slow)).clamp(0, 1)
    return f * kept + f / factor * (1 - kept)


def _rotary(x, positions, frequencies, interleaved, magnitude, out, inverse):
    d = _dtype("x", x.dtype)
    hx = _heads("x", x)
    rows, heads, dim = x.shape
    p, wide = _index("positions", positions, rows, x)
    if frequencies.dim() != 1:
        _refuse(f"frequencies is {tuple(frequencies.shape)}, (turned / 2,) is wanted")
    f = _vector("frequencies", frequencies, frequencies.shape[0], torch.float64, x)
    if out is None:
        y = x.new_empty(rows, heads, dim)
        hy = y.data_ptr(), heads * dim, dim
    else:
        y, hy = out, _heads("out", out, x, rows, heads, dim)
    _check(load().pase_rotary(d, rows, heads, dim, 2 * frequencies.shape[0], bool(interleaved), inverse, *hx, p, wide, f,
                              magnitude, *hy, _raw_stream(x.get_device())))
    _written(out)
    return y


@_on_device("x")
def rotary_forward(x, positions, frequencies, interleaved: bool = False, magnitude: float = 1.0, out=None):
    """Turns pair i of every head of row t by the angle positions[t] * frequencies[i], times magnitude.

    x: [rows, heads, dim], rows and heads as for attention; positions: [rows], int32 or
    int64; frequencies: float64 [turned / 2] (`rotary_frequencies`).  Pairs are elements i and i + turned / 2,
    or (interleaved) 2 i and 2 i + 1; the elements from `turned` on stay.  out may be x, or a tensor with no element of x."""
    return _rotary(x, positions, frequencies, interleaved, magnitude, out, 0)


@_on_device("dy")
def rotary_backward(dy, positions, frequencies, interleaved: bool = False, magnitude: float = 1.0, out=None):
    """dx of `rotary_forward`: the same turned the other way.  out may be dy, or a tensor with no element of it."""
    return _rotary(dy, positions, frequencies, interleaved, magnitude, out, 1)


# ------------------------------------------------------------------ dropout
def _dropout(x, p, seed, residual):
    d = _dtype("x", x.dtype)
    ldx = _matrix("x", x)
    rows, width = x.shape
    r, ldr = None, 0
    if residual is not None:
        ldr, r = _matrix("residual", residual, x, rows, width), residual.data_ptr()
    s = _vector("seed", seed, 2, torch.int64, x)
    y = x.new_empty(rows, width)
    _check(load().pase_dropout(d, rows, width, x.data_ptr(), ldx, r, ldr, p, s, y.data_ptr(), width, _raw_stream(x.get_device())))
    return y


@_on_device("x")
def dropout_forward(x, p: float, seed, residual=None):
    """residual + keep * x / (1 - p) for x [rows, width], where every element is kept with
    probability 1 - p (p to the nearest multiple of 2 ** -16).  Which are kept follows from seed, two int64 on the device, and the
    element's row and column alone: no mask is stored.  Calls whose masks are to be
    independent need different seeds; a captured call reads its seed when it is replayed."""
    return _dropout(x, p, seed, residual)


@_on_device("dy")
def dropout_backward(dy, p: float, seed):
    """dx of `dropout_forward` with the same p and seed; the residual's gradient is dy."""
    return _dropout(dy, p, seed, None)


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


def _heads_adjacent(t):
    """The same for [rows, heads, dim], whose rows may also be further apart than the operators take."""
    rows, heads, dim = t.shape
    ld, hs, step = t.stride()
    return t if step == 1 and (rows < 2 or dim <= ld <= MAX_ROW_STRIDE) and (heads < 2 or hs >= dim) else t.contiguous()


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


class _Attention(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, v, q_offsets, k_offsets, k_lengths, causal, scale):
        out, lse = attention_forward(q, k, v, q_offsets, k_offsets, k_lengths, causal, scale)
        ctx.save_for_backward(q, k, v, out, lse, q_offsets, k_offsets, k_lengths)
        ctx.rest = causal, scale
        return out

    @staticmethod
    @once_differentiable
    def backward(ctx, dout):
        q, k, v, out, lse, q_offsets, k_offsets, k_lengths = ctx.saved_tensors
        grads = attention_backward(_heads_adjacent(dout), q, k, v, out, lse, q_offsets, k_offsets, k_lengths, *ctx.rest)
        return *grads, None, None, None, None, None


def attention(q, k, v, q_offsets, k_offsets, k_lengths=None, causal: bool = False, scale=None):
    """The out of `attention_forward`, differentiable in q, k and v."""
    return _Attention.apply(q, k, v, q_offsets, k_offsets, k_lengths, causal, scale)


class _Rotary(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, positions, frequencies, interleaved, magnitude):
        ctx.save_for_backward(positions, frequencies)
        ctx.rest = interleaved, magnitude
        return rotary_forward(x, positions, frequencies, interleaved, magnitude)

    @staticmethod
    @once_differentiable
    def backward(ctx, dy):
        return rotary_backward(_heads_adjacent(dy), *ctx.saved_tensors, *ctx.rest), None, None, None, None


def rotary(x, positions, frequencies, interleaved: bool = False, magnitude: float = 1.0):
    """`rotary_forward`, differentiable in x."""
    return _Rotary.apply(x, positions, frequencies, interleaved, magnitude)


class _Dropout(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, p, seed, residual):
        # the seed as it is now: a caller may advance it in place before the backward pass
        ctx.save_for_backward(seed.clone())
        ctx.p = p
        return dropout_forward(x, p, seed, residual)

    @staticmethod
    @once_differentiable
    def backward(ctx, dy):
        seed, = ctx.saved_tensors
        dx = dropout_backward(_rows_adjacent(dy), ctx.p, seed) if ctx.needs_input_grad[0] else None
        return dx, None, None, dy if ctx.needs_input_grad[3] else None


def dropout(x, p: float, seed, residual=None):
    """`dropout_forward`, differentiable in x and residual."""
    return _Dropout.apply(x, p, seed, residual)


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

"""Operators of a model whose gradients the engine's caller passes in (`GRAD_EXTERNAL`).

The engine takes `ext[n][d]`: the gradient of every worker at the same x.  These are the layers of a model whose
backward pass leaves them, each worker's (or each expert's) own: rows are split into groups by `offsets`, and
gradients of weights come out by group, written where the caller wants them (a view of `ext`, for instance).

    group_matmul, group_matmul_dx, group_matmul_dw    products of ragged groups of rows with a matrix for each
    layer_norm, layer_norm_backward                   gradients of weight and bias by group
    dropout                                           from the counter-based generator; no mask is stored
    preference_loss, preference_loss_backward         logistic loss of paired sequences' log ratios, from logits

Argument marshalling only: every function checks what the library cannot see (devices, types, shapes, strides),
enqueues on the current stream of its tensors' device and returns without waiting.  Nothing is recorded for automatic
differentiation.  Tensors are float32, bfloat16 or float16 on one GPU, unit stride inside a row; `offsets` is an int64
tensor on the same GPU, ascending, and is not read by the host.  Rows that belong to no group are left as they are in
outputs passed by the caller and unspecified in those made here.  include/adacgd.h has the definitions.
"""
from __future__ import annotations

import ctypes as C
import functools
import struct

import torch

from .engine import AdaCGDError, load_library

FORWARD, DX, DW = 0, 1, 2


class Tensor(C.Structure):
    """adacgd_tensor."""
    _fields_ = [("data", C.c_void_p), ("dtype", C.c_int32), ("pad", C.c_int32), ("stride", C.c_int64), ("group_stride", C.c_int64)]


# (descriptors are passed as the bytes of an adacgd_tensor: a small call takes as long as the host needs to make it)
_tensor = struct.Struct("Piiqq").pack
_DTYPES = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}

_P, _I64, _I32, _D = C.c_void_p, C.c_int64, C.c_int32, C.c_double
ARGTYPES = {
    "adacgd_group_matmul_workspace_bytes": [_I32, _I32, _I64, _I64, _I64, _I64, _P],
    "adacgd_group_matmul": [_I32, _I64, _I64, _I64, _I64, _P, _P, _P, _P, _P, _I64, _P],
    "adacgd_layer_norm": [_I64, _I64, _P, _P, _P, _D, _P, _P, _P, _P],
    "adacgd_layer_norm_backward_workspace_bytes": [_I64, _I64, _I64, _P],
    "adacgd_layer_norm_backward": [_I64, _I64, _I64, _P, _P, _P, _P, _P, _P, _P, _P, _P, _P, _I64, _P],
    "adacgd_dropout": [_I64, _I64, _P, _P, _P, _D, C.c_uint64, C.c_uint32, _P, C.c_uint32, C.c_uint64, _P],
    "adacgd_preference_loss_workspace_bytes": [_I64, _I64, _I64, _P],
    "adacgd_preference_loss": [_I64, _I64, _I64, _P, _P, _P, _P, _D, _D, _P, _P, _P, _P, _P, _I64, _P],
    "adacgd_preference_loss_backward": [_I64, _I64, _I64, _P, _P, _P, _P, _P, _P, _D, _D, _P, _P],
}

_lib = None


def _library():
    global _lib
    if _lib is None:
        lib = load_library()
        for name, types in ARGTYPES.items():
            f = getattr(lib, name)
            f.argtypes, f.restype = types, C.c_int
        _lib = lib
    return _lib


def _fail(rc):
    raise AdaCGDError(rc, _library().adacgd_last_error(None).decode())


def _call(like, f, *args):
    """Enqueues on the current stream of the device of `like`, whichever device is current."""
    index = like.get_device()
    if index == torch.cuda.current_device():
        rc = f(*args, torch._C._cuda_getCurrentRawStream(index))
    else:
        with torch.cuda.device(index):
            rc = f(*args, torch._C._cuda_getCurrentRawStream(index))
    if rc:
        _fail(rc)


def _refuse(text, *args):
    raise ValueError(text % args)


def _matrix(name, t, rows, columns, like=None, groups=None):
    """The descriptor of a [rows, columns] (or [groups, rows, columns]) tensor."""
    if t.shape != ((rows, columns) if groups is None else (groups, rows, columns)):
        _refuse("%s: shape %s expected, got %s", name, (rows, columns) if groups is None else (groups, rows, columns), tuple(t.shape))
    if not t.is_cuda:
        _refuse("%s is not on a GPU", name)
    if like is not None and t.get_device() != like.get_device():
        _refuse("%s is on another device", name)
    strides = t.stride()
    if strides[-1] != 1 and columns > 1:
        _refuse("%s: unit stride inside a row expected", name)
    dtype = _DTYPES.get(t.dtype)
    if dtype is None:
        raise TypeError("%s: float32, bfloat16 or float16 expected, got %s" % (name, t.dtype))
    return _tensor(t.data_ptr(), dtype, 0, strides[-2], 0 if groups is None else strides[0])


def _vector(name, t, length, dtype, like):
    if t.shape != (length,):
        _refuse("%s: shape (%s,) expected, got %s", name, length, tuple(t.shape))
    if not t.is_cuda or t.get_device() != like.get_device():
        _refuse("%s is on another device", name)
    if t.dtype != dtype:
        _refuse("%s: %s expected, got %s", name, dtype, t.dtype)
    if length > 1 and t.stride(0) != 1:
        _refuse("%s is not contiguous", name)
    return t.data_ptr()


def _offsets(t, like):
    if t.dim() != 1 or t.numel() < 1:
        _refuse("offsets: groups + 1 row numbers expected")
    return _vector("offsets", t, t.numel(), torch.int64, like)


@functools.lru_cache(maxsize=256)
def _bytes(name, *args):
    n = C.c_int64(0)
    rc = getattr(_library(), name)(*args, C.addressof(n))
    if rc:
        _fail(rc)
    return n.value


def _workspace(like, name, *args):
    """(tensor to keep, its address, its size): torch's allocator owns it, on the stream that the call is enqueued on."""
    size = _bytes(name, *args)
    if size == 0:
        return None, None, 0
    w = like.new_empty(size, dtype=torch.uint8)
    return w, w.data_ptr(), size


def _gpu(name, t, dims):
    if t.dim() != dims:
        _refuse("%s: %d dimensions expected, got %s", name, dims, tuple(t.shape))
    if not t.is_cuda:
        _refuse("%s is not on a GPU", name)


def _product(product, a, b, offsets, out, out_dtype):
    lib = _library()
    _gpu("the first argument", a, 2)
    _gpu("the second argument", b, 2 if product == DW else 3)
    off, groups = _offsets(offsets, a), offsets.numel() - 1
    rows = a.shape[0]
    if product == DW:
        n, k = a.shape[1], b.shape[1]
        ta, tb, shape = _matrix("the first argument", a, rows, n), _matrix("the second argument", b, rows, k, a), (groups, n, k)
    else:
        _, n, k = b.shape
        ta, tb = _matrix("the first argument", a, rows, k if product == FORWARD else n), _matrix("the weights", b, n, k, a, groups)
        shape = (rows, n if product == FORWARD else k)
    if out is None:
        out = a.new_empty(shape, dtype=out_dtype)
    tc = _matrix("out", out, shape[-2], shape[-1], a, groups if product == DW else None)
    keep, ws, size = _workspace(a, "adacgd_group_matmul_workspace_bytes", product, _DTYPES[a.dtype], rows, groups, n, k) if product == DW else (None, None, 0)
    _call(a, lib.adacgd_group_matmul, product, rows, groups, n, k, off, ta, tb, tc, ws, size)
    return out


def group_matmul(x, w, offsets, out=None):
    """out[r] = w[g] x[r] for the rows r of group g: x [rows, k], w [groups, n, k], out [rows, n] of x's type or float32.
    w may be an expanded view of one matrix for all groups."""
    return _product(FORWARD, x, w, offsets, out, x.dtype)


def group_matmul_dx(dy, w, offsets, out=None):
    """out[r] = w[g]^T dy[r]: the gradient of `group_matmul`'s rows.  dy [rows, n], out [rows, k] of dy's type or float32."""
    return _product(DX, dy, w, offsets, out, dy.dtype)


def group_matmul_dw(dy, x, offsets, out=None):
    """out[g] = sum over the rows of g of dy[r] x[r]^T: each group's own gradient of the weights, also where all groups
    share them.  dy [rows, n], x [rows, k], out [groups, n, k] float32 (or of x's type; rows and matrices any distance apart)."""
    return _product(DW, dy, x, offsets, out, torch.float32)


def layer_norm(x, weight=None, bias=None, eps=1e-5, out=None, statistics=True):
    """(y, mean, rstd) of the rows of x [rows, d]: y = (x - mean) rstd weight + bias, rstd = 1 / sqrt(var + eps).
    weight, bias: float32 [d].  `statistics` false: mean and rstd are not kept and come back as None.  out may be x."""
    _gpu("x", x, 2)
    rows, d = x.shape
    tx = _matrix("x", x, rows, d)
    w = None if weight is None else _vector("weight", weight, d, torch.float32, x)
    b = None if bias is None else _vector("bias", bias, d, torch.float32, x)
    if out is None:
        out = x.new_empty((rows, d))
    to = _matrix("out", out, rows, d, x)
    mean, rstd = x.new_empty((2, rows), dtype=torch.float32).unbind() if statistics else (None, None)
    _call(x, _library().adacgd_layer_norm, rows, d, tx, w, b, eps, to, mean.data_ptr() if statistics else None,
          rstd.data_ptr() if statistics else None)
    return out, mean, rstd


def layer_norm_backward(dy, x, weight, mean, rstd, offsets=None, dx=None, dweight=None, dbias=None):
    """(dx, dweight, dbias) of `layer_norm`: dx [rows, d] of x's type; dweight, dbias [groups, d] float32, summed over each
    group's own rows (offsets None: one group of all rows)."""
    _gpu("x", x, 2)
    rows, d = x.shape
    off, groups = (None, 1) if offsets is None else (_offsets(offsets, x), offsets.numel() - 1)
    tx, tdy = _matrix("x", x, rows, d), _matrix("dy", dy, rows, d, x)
    w = None if weight is None else _vector("weight", weight, d, torch.float32, x)
    m, r = _vector("mean", mean, rows, torch.float32, x), _vector("rstd", rstd, rows, torch.float32, x)
    dx = x.new_empty((rows, d)) if dx is None else dx
    dweight = x.new_empty((groups, d), dtype=torch.float32) if dweight is None else dweight
    dbias = x.new_empty((groups, d), dtype=torch.float32) if dbias is None else dbias
    tdx, tdw, tdb = _matrix("dx", dx, rows, d, x), _matrix("dweight", dweight, groups, d, x), _matrix("dbias", dbias, groups, d, x)
    keep, ws, size = _workspace(x, "adacgd_layer_norm_backward_workspace_bytes", rows, groups, d)
    _call(x, _library().adacgd_layer_norm_backward, rows, groups, d, off, tdy, tx, w, m, r, tdx, tdw, tdb, ws, size)
    return dx, dweight, dbias


def dropout(x, p, seed, step=0, layer=0, first=0, residual=None, out=None):
    """residual + x / (1 - p) where an element is kept, residual (or 0) where it is dropped; x [rows, d].

    What is kept depends on (seed, step, layer, first + position) only: the backward pass is the same call on the gradient,
    without the residual.  step: a number, or a one-element int64 tensor on the GPU that a captured call reads anew at every
    replay.  Pieces of a batch drawn one by one take their first element's position in it as `first`.  out may be x or residual."""
    _gpu("x", x, 2)
    rows, d = x.shape
    tx = _matrix("x", x, rows, d)
    tr = None if residual is None else _matrix("residual", residual, rows, d, x)
    if out is None:
        out = x.new_empty((rows, d))
    to = _matrix("out", out, rows, d, x)
    step_dev = None
    if isinstance(step, torch.Tensor):
        step_dev, step = _vector("step", step.reshape(-1), 1, torch.int64, x), 0
    if not (0 <= step < 1 << 32 and 0 <= layer < (1 << 32) - 1):
        _refuse("step and layer must fit 32 bits (layer below 2^32 - 1)")
    if not (0 <= seed < 1 << 64 and 0 <= first < 1 << 64):
        _refuse("seed and first must fit 64 bits")
    _call(x, _library().adacgd_dropout, rows, d, tx, tr, to, p, seed, step, step_dev, layer, first)
    return out


def preference_loss(logits, targets, offsets, ref=None, beta=0.1, smoothing=0.0):
    """(loss [pairs], margin [pairs], logp [tokens], lse [tokens]), all float32, of 2 pairs sequences of token rows.

    Sequence 2p is pair p's preferred one.  logits [tokens, v], targets [tokens] int64 (outside [0, v): the token does not
    count), ref [tokens] float32: the reference model's logp.  margin = sum of (logp - ref) over the one minus the other;
    loss = log(1 + exp(-beta margin)), or with label smoothing s, (1 - s) of that and s of log(1 + exp(beta margin))."""
    _gpu("logits", logits, 2)
    tokens, v = logits.shape
    off = _offsets(offsets, logits)
    if offsets.numel() % 2 == 0:
        _refuse("offsets: an even number of sequences expected")
    pairs = (offsets.numel() - 1) // 2
    tl = _matrix("logits", logits, tokens, v)
    tg = _vector("targets", targets, tokens, torch.int64, logits)
    rf = None if ref is None else _vector("ref", ref, tokens, torch.float32, logits)
    loss, margin = logits.new_empty((2, pairs), dtype=torch.float32).unbind()
    logp, lse = logits.new_empty((2, tokens), dtype=torch.float32).unbind()
    keep, ws, size = _workspace(logits, "adacgd_preference_loss_workspace_bytes", tokens, pairs, v)
    _call(logits, _library().adacgd_preference_loss, tokens, pairs, v, tl, tg, off, rf, beta, smoothing, loss.data_ptr(),
          margin.data_ptr(), logp.data_ptr(), lse.data_ptr(), ws, size)
    return loss, margin, logp, lse


def preference_loss_backward(dloss, logits, targets, offsets, margin, lse, beta=0.1, smoothing=0.0, out=None):
    """The gradient of sum(dloss * loss) by logits, [tokens, v] of logits' type; out may be logits."""
    _gpu("logits", logits, 2)
    tokens, v = logits.shape
    off = _offsets(offsets, logits)
    if offsets.numel() % 2 == 0:
        _refuse("offsets: an even number of sequences expected")
    pairs = (offsets.numel() - 1) // 2
    tl = _matrix("logits", logits, tokens, v)
    tg = _vector("targets", targets, tokens, torch.int64, logits)
    dl, mg = _vector("dloss", dloss, pairs, torch.float32, logits), _vector("margin", margin, pairs, torch.float32, logits)
    ls = _vector("lse", lse, tokens, torch.float32, logits)
    if out is None:
        out = logits.new_empty((tokens, v))
    to = _matrix("out", out, tokens, v, logits)
    _call(logits, _library().adacgd_preference_loss_backward, tokens, pairs, v, dl, tl, tg, off, mg, ls, beta, smoothing, to)
    return out

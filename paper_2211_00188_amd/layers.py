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

from .engine import AdaCGDError, load_library

FORWARD, DX, DW = 0, 1, 2


class Tensor(C.Structure):
    _fields_ = [("data", C.c_void_p), ("dtype", C.c_int32), ("pad", C.c_int32), ("stride", C.c_int64), ("group_stride", C.c_int64)]


_P, _I64, _I32, _D, _T = C.c_void_p, C.c_int64, C.c_int32, C.c_double, C.POINTER(Tensor)
ARGTYPES = {
    "adacgd_group_matmul_workspace_bytes": [_I32, _I32, _I64, _I64, _I64, _I64, C.POINTER(_I64)],
    "adacgd_group_matmul": [_I32, _I64, _I64, _I64, _I64, _P, _T, _T, _T, _P, _I64, _P],
    "adacgd_layer_norm": [_I64, _I64, _T, _P, _P, _D, _T, _P, _P, _P],
    "adacgd_layer_norm_backward_workspace_bytes": [_I64, _I64, _I64, C.POINTER(_I64)],
    "adacgd_layer_norm_backward": [_I64, _I64, _I64, _P, _T, _T, _P, _P, _P, _T, _T, _T, _P, _I64, _P],
    "adacgd_dropout": [_I64, _I64, _T, _T, _T, _D, C.c_uint64, C.c_uint32, _P, C.c_uint32, C.c_uint64, _P],
    "adacgd_preference_loss_workspace_bytes": [_I64, _I64, _I64, C.POINTER(_I64)],
    "adacgd_preference_loss": [_I64, _I64, _I64, _T, _P, _P, _P, _D, _D, _P, _P, _P, _P, _P, _I64, _P],
    "adacgd_preference_loss_backward": [_I64, _I64, _I64, _P, _T, _P, _P, _P, _P, _D, _D, _T, _P],
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


def _call(device, name, *args):
    """Enqueues on `device`'s current stream, whichever device is current."""
    import torch
    lib = _library()
    with torch.cuda.device(device):
        rc = getattr(lib, name)(*args, torch.cuda.current_stream(device).cuda_stream)
    if rc:
        raise AdaCGDError(rc, lib.adacgd_last_error(None).decode())


def _dtype(t):
    import torch
    try:
        return {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}[t.dtype]
    except KeyError:
        raise TypeError("float32, bfloat16 or float16 expected, got %s" % t.dtype) from None


def _check(cond, text, *args):
    if not cond:
        raise ValueError(text % args)


def _matrix(name, t, rows, columns, like=None, groups=None):
    """The descriptor of a [rows, columns] (or [groups, rows, columns]) tensor."""
    shape = (rows, columns) if groups is None else (groups, rows, columns)
    _check(tuple(t.shape) == shape, "%s: shape %s expected, got %s", name, shape, tuple(t.shape))
    _check(t.is_cuda, "%s is not on a GPU", name)
    _check(like is None or t.device == like.device, "%s is on another device", name)
    _check(columns <= 1 or t.stride(-1) == 1, "%s: unit stride inside a row expected", name)
    return Tensor(t.data_ptr(), _dtype(t), 0, t.stride(-2), 0 if groups is None else t.stride(0))


def _vector(name, t, length, dtype, like):
    _check(tuple(t.shape) == (length,), "%s: shape (%s,) expected, got %s", name, length, tuple(t.shape))
    _check(t.device == like.device, "%s is on another device", name)
    _check(t.dtype == dtype, "%s: %s expected, got %s", name, dtype, t.dtype)
    _check(length <= 1 or t.stride(0) == 1, "%s is not contiguous", name)
    return t.data_ptr()


def _offsets(t, like, groups=None):
    import torch
    _check(t.dim() == 1 and t.numel() >= 1, "offsets: groups + 1 row numbers expected")
    return _vector("offsets", t, t.numel() if groups is None else groups + 1, torch.int64, like)


def _workspace(name, device, *args):
    import torch
    n = C.c_int64(0)
    rc = getattr(_library(), name)(*args, C.byref(n))
    if rc:
        raise AdaCGDError(rc, _library().adacgd_last_error(None).decode())
    if n.value == 0:
        return None, None, 0
    w = torch.empty(n.value, dtype=torch.uint8, device=device)
    return w, w.data_ptr(), n.value


def _gpu(name, t, dims):
    _check(t.dim() == dims, "%s: %d dimensions expected, got %s", name, dims, tuple(t.shape))
    _check(t.is_cuda, "%s is not on a GPU", name)


def _product(product, a, b, offsets, out, out_dtype):
    import torch
    _gpu("the first argument", a, 2)
    _gpu("the second argument", b, 2 if product == DW else 3)
    groups = offsets.numel() - 1
    rows = a.shape[0]
    n, k = (a.shape[1], b.shape[1]) if product == DW else (b.shape[1], b.shape[2])
    off = _offsets(offsets, a)
    ta = _matrix("the first argument", a, rows, k if product == FORWARD else n)
    if product == DW:
        tb = _matrix("the second argument", b, rows, k, a)
        shape = (groups, n, k)
    else:
        tb = _matrix("the weights", b, n, k, a, groups)
        shape = (rows, n if product == FORWARD else k)
    if out is None:
        out = torch.empty(shape, dtype=out_dtype, device=a.device)
    tc = _matrix("out", out, shape[-2], shape[-1], a, groups if product == DW else None)
    keep, ws, size = _workspace("adacgd_group_matmul_workspace_bytes", a.device, product, ta.dtype, rows, groups, n, k)
    _call(a.device, "adacgd_group_matmul", product, rows, groups, n, k, off, ta, tb, tc, ws, size)
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
    import torch
    return _product(DW, dy, x, offsets, out, torch.float32)


def layer_norm(x, weight=None, bias=None, eps=1e-5, out=None, statistics=True):
    """(y, mean, rstd) of the rows of x [rows, d]: y = (x - mean) rstd weight + bias, rstd = 1 / sqrt(var + eps).
    weight, bias: float32 [d].  `statistics` false: mean and rstd are not kept and come back as None.  out may be x."""
    import torch
    _gpu("x", x, 2)
    rows, d = x.shape
    tx = _matrix("x", x, rows, d)
    w = None if weight is None else _vector("weight", weight, d, torch.float32, x)
    b = None if bias is None else _vector("bias", bias, d, torch.float32, x)
    if out is None:
        out = torch.empty((rows, d), dtype=x.dtype, device=x.device)
    to = _matrix("out", out, rows, d, x)
    mean = torch.empty(rows, dtype=torch.float32, device=x.device) if statistics else None
    rstd = torch.empty(rows, dtype=torch.float32, device=x.device) if statistics else None
    _call(x.device, "adacgd_layer_norm", rows, d, tx, w, b, float(eps), to, mean.data_ptr() if statistics else None,
          rstd.data_ptr() if statistics else None)
    return out, mean, rstd


def layer_norm_backward(dy, x, weight, mean, rstd, offsets=None, dx=None, dweight=None, dbias=None):
    """(dx, dweight, dbias) of `layer_norm`: dx [rows, d] of x's type; dweight, dbias [groups, d] float32, summed over each
    group's own rows (offsets None: one group of all rows)."""
    import torch
    _gpu("x", x, 2)
    rows, d = x.shape
    off, groups = (None, 1) if offsets is None else (_offsets(offsets, x), offsets.numel() - 1)
    tx, tdy = _matrix("x", x, rows, d), _matrix("dy", dy, rows, d, x)
    w = None if weight is None else _vector("weight", weight, d, torch.float32, x)
    m, r = _vector("mean", mean, rows, torch.float32, x), _vector("rstd", rstd, rows, torch.float32, x)
    dx = torch.empty((rows, d), dtype=x.dtype, device=x.device) if dx is None else dx
    dweight = torch.empty((groups, d), dtype=torch.float32, device=x.device) if dweight is None else dweight
    dbias = torch.empty((groups, d), dtype=torch.float32, device=x.device) if dbias is None else dbias
    tdx, tdw, tdb = _matrix("dx", dx, rows, d, x), _matrix("dweight", dweight, groups, d, x), _matrix("dbias", dbias, groups, d, x)
    keep, ws, size = _workspace("adacgd_layer_norm_backward_workspace_bytes", x.device, rows, groups, d)
    _call(x.device, "adacgd_layer_norm_backward", rows, groups, d, off, tdy, tx, w, m, r, tdx, tdw, tdb, ws, size)
    return dx, dweight, dbias


def dropout(x, p, seed, step=0, layer=0, first=0, residual=None, out=None):
    """residual + x / (1 - p) where an element is kept, residual (or 0) where it is dropped; x [rows, d].

    What is kept depends on (seed, step, layer, first + position) only: the backward pass is the same call on the gradient,
    without the residual.  step: a number, or a one-element int64 tensor on the GPU that a captured call reads anew at every
    replay.  Pieces of a batch drawn one by one take their first element's position in it as `first`.  out may be x or residual."""
    import torch
    _gpu("x", x, 2)
    rows, d = x.shape
    tx = _matrix("x", x, rows, d)
    tr = None if residual is None else _matrix("residual", residual, rows, d, x)
    if out is None:
        out = torch.empty((rows, d), dtype=x.dtype, device=x.device)
    to = _matrix("out", out, rows, d, x)
    step_dev = None
    if isinstance(step, torch.Tensor):
        step_dev, step = _vector("step", step.reshape(-1), 1, torch.int64, x), 0
    _check(0 <= step < 1 << 32 and 0 <= layer < (1 << 32) - 1, "step and layer must fit 32 bits (layer below 2^32 - 1)")
    _check(0 <= seed < 1 << 64 and 0 <= first < 1 << 64, "seed and first must fit 64 bits")
    _call(x.device, "adacgd_dropout", rows, d, tx, tr, to, float(p), seed, step, step_dev, layer, first)
    return out


def preference_loss(logits, targets, offsets, ref=None, beta=0.1, smoothing=0.0):
    """(loss [pairs], margin [pairs], logp [tokens], lse [tokens]), all float32, of 2 pairs sequences of token rows.

    Sequence 2p is pair p's preferred one.  logits [tokens, v], targets [tokens] int64 (outside [0, v): the token does not
    count), ref [tokens] float32: the reference model's logp.  margin = sum of (logp - ref) over the one minus the other;
    loss = log(1 + exp(-beta margin)), or with label smoothing s, (1 - s) of that and s of log(1 + exp(beta margin))."""
    import torch
    _gpu("logits", logits, 2)
    tokens, v = logits.shape
    off = _offsets(offsets, logits)
    _check(offsets.numel() % 2 == 1, "offsets: an even number of sequences expected")
    pairs = (offsets.numel() - 1) // 2
    tl = _matrix("logits", logits, tokens, v)
    tg = _vector("targets", targets, tokens, torch.int64, logits)
    rf = None if ref is None else _vector("ref", ref, tokens, torch.float32, logits)
    loss, margin = (torch.empty(pairs, dtype=torch.float32, device=logits.device) for _ in range(2))
    logp, lse = (torch.empty(tokens, dtype=torch.float32, device=logits.device) for _ in range(2))
    keep, ws, size = _workspace("adacgd_preference_loss_workspace_bytes", logits.device, tokens, pairs, v)
    _call(logits.device, "adacgd_preference_loss", tokens, pairs, v, tl, tg, off, rf, float(beta), float(smoothing), loss.data_ptr(),
          margin.data_ptr(), logp.data_ptr(), lse.data_ptr(), ws, size)
    return loss, margin, logp, lse


def preference_loss_backward(dloss, logits, targets, offsets, margin, lse, beta=0.1, smoothing=0.0, out=None):
    """The gradient of sum(dloss * loss) by logits, [tokens, v] of logits' type; out may be logits."""
    import torch
    _gpu("logits", logits, 2)
    tokens, v = logits.shape
    off = _offsets(offsets, logits)
    _check(offsets.numel() % 2 == 1, "offsets: an even number of sequences expected")
    pairs = (offsets.numel() - 1) // 2
    tl = _matrix("logits", logits, tokens, v)
    tg = _vector("targets", targets, tokens, torch.int64, logits)
    dl, mg = _vector("dloss", dloss, pairs, torch.float32, logits), _vector("margin", margin, pairs, torch.float32, logits)
    ls = _vector("lse", lse, tokens, torch.float32, logits)
    if out is None:
        out = torch.empty((tokens, v), dtype=logits.dtype, device=logits.device)
    to = _matrix("out", out, tokens, v, logits)
    _call(logits.device, "adacgd_preference_loss_backward", tokens, pairs, v, dl, tl, tg, off, mg, ls, float(beta), float(smoothing), to)
    return out

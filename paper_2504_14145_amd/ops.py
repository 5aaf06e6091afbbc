"""Python binding of the stage operators (include/dip_ops.h).

The operators that the cost tables price -- matrix product with its epilogue,
dropout whose mask is never stored, group norm (layer norm) with an activation
-- forward and their gradients, as HIP kernels of ``libdip_sim.so``.  Functions
take torch device tensors (the last dimension contiguous, other strides free),
check them, and enqueue on ``stream`` (torch's current one by default).  As in
the rest of the package PyTorch provides device memory and the stream, nothing
else: outputs and workspaces come from its allocator where none is given, and
no call records an autograd graph.
"""
from __future__ import annotations

import ctypes

from . import E_CAPACITY, _check, load

F32, F16, BF16 = 0, 1, 2
ACTS = {"none": 0, "relu": 1, "silu": 2, "gelu": 3}

EXPORTS = ("dip_linear_workspace", "dip_linear", "dip_linear_grad_workspace", "dip_linear_grad",
           "dip_dropout_add", "dip_group_norm_workspace", "dip_group_norm",
           "dip_group_norm_grad_workspace", "dip_group_norm_grad")

_vp, _i32, _i64 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64


class Dropout(ctypes.Structure):
    """Dropout of probability ``p`` (rounded to 65536ths, below 1).  The mask is
    a function of (seed, offset, row0 + row, column): the same object gives the
    same mask in the forward, the gradient and a recomputed forward, and a piece
    of a sample that starts at its row ``row0`` draws the sample's mask."""
    _fields_ = [("seed", ctypes.c_uint64), ("offset", ctypes.c_uint64),
                ("row0", ctypes.c_uint32), ("drop_of", ctypes.c_uint32)]

    def __init__(self, p: float, seed: int, offset: int = 0, row0: int = 0):
        if not 0.0 <= p < 1.0:
            raise ValueError(f"dropout probability {p} is not in [0, 1)")
        if not 0 <= row0 < 1 << 32:
            raise ValueError(f"row0 {row0} is not in [0, 2^32)")
        mask = (1 << 64) - 1
        super().__init__(int(seed) & mask, int(offset) & mask, int(row0),
                         min(65535, round(65536 * p)))

    @property
    def scale(self) -> float:
        """What kept elements are multiplied by."""
        return 65536.0 / (65536 - self.drop_of)


class _Linear(ctypes.Structure):
    _fields_ = [("m", _i64), ("n", _i64), ("k", _i64), ("dtype", _i32), ("act", _i32),
                ("x", _vp), ("ldx", _i64), ("w", _vp), ("ldw", _i64), ("bias", _vp),
                ("residual", _vp), ("ldr", _i64), ("drop", Dropout), ("y", _vp), ("ldy", _i64),
                ("pre", _vp), ("ldp", _i64), ("workspace", _vp), ("workspace_bytes", _i64)]


class _LinearGrad(ctypes.Structure):
    _fields_ = [("m", _i64), ("n", _i64), ("k", _i64), ("dtype", _i32), ("act", _i32),
                ("dy", _vp), ("ldy", _i64), ("x", _vp), ("ldx", _i64), ("w", _vp), ("ldw", _i64),
                ("pre", _vp), ("ldp", _i64), ("drop", Dropout), ("dx", _vp), ("lddx", _i64),
                ("dw", _vp), ("lddw", _i64), ("db", _vp), ("grad_dtype", _i32),
                ("accumulate", _i32), ("workspace", _vp), ("workspace_bytes", _i64)]


class _GroupNorm(ctypes.Structure):
    _fields_ = [("b", _i64), ("s", _i64), ("c", _i64), ("groups", _i32), ("dtype", _i32),
                ("act", _i32), ("eps", ctypes.c_float), ("x", _vp), ("x_sb", _i64),
                ("x_ss", _i64), ("gamma", _vp), ("beta", _vp), ("y", _vp), ("y_sb", _i64),
                ("y_ss", _i64), ("mean", _vp), ("rstd", _vp), ("workspace", _vp),
                ("workspace_bytes", _i64)]


class _GroupNormGrad(ctypes.Structure):
    _fields_ = [("b", _i64), ("s", _i64), ("c", _i64), ("groups", _i32), ("dtype", _i32),
                ("act", _i32), ("dy", _vp), ("dy_sb", _i64), ("dy_ss", _i64), ("x", _vp),
                ("x_sb", _i64), ("x_ss", _i64), ("gamma", _vp), ("beta", _vp), ("mean", _vp),
                ("rstd", _vp), ("dx", _vp), ("dx_sb", _i64), ("dx_ss", _i64), ("dgamma", _vp),
                ("dbeta", _vp), ("workspace", _vp), ("workspace_bytes", _i64)]


_lib = None
_torch = None
_raw_stream = None   # device index -> handle of torch's current stream
_types = {}


def _load():
    """The library with the operators' signatures, and torch."""
    global _lib, _torch, _raw_stream
    if _lib is None:
        import torch
        lib = load()
        for name, args in (("dip_linear", _Linear), ("dip_linear_grad", _LinearGrad),
                           ("dip_group_norm", _GroupNorm),
                           ("dip_group_norm_grad", _GroupNormGrad)):
            getattr(lib, name).argtypes = [ctypes.POINTER(args), _vp]
            getattr(lib, name).restype = ctypes.c_int
            getattr(lib, name + "_workspace").argtypes = [ctypes.POINTER(args)]
            getattr(lib, name + "_workspace").restype = _i64
        lib.dip_dropout_add.argtypes = [_i32, _i64, _i64, _vp, _i64, _vp, _i64,
                                        ctypes.POINTER(Dropout), _vp, _i64, _vp]
        lib.dip_dropout_add.restype = ctypes.c_int
        _types.update({torch.float32: F32, torch.float16: F16, torch.bfloat16: BF16})
        _raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream",
                              lambda index: torch.cuda.current_stream(index).cuda_stream)
        _torch, _lib = torch, lib
    return _lib


_NO_DROP = Dropout(0.0, 0)


def _need(ok: bool, what: str):
    if not ok:
        raise ValueError(what)


def _act(name) -> int:
    code = ACTS.get(name)
    if code is None:
        raise ValueError(f"unknown activation {name!r}: one of {', '.join(ACTS)}")
    return code


def _refuse(t, shape, dtype, device, name):
    if not isinstance(t, _torch.Tensor):
        raise ValueError(f"{name}: want a tensor, got {type(t).__name__}")
    if t.shape != shape or t.dtype != dtype or t.device != device:
        raise ValueError(f"{name}: want {tuple(shape)} {dtype} on {device}, got {tuple(t.shape)} {t.dtype} on {t.device}")
    raise ValueError(f"{name}: the last dimension has to be contiguous")


_NONE = (None, 0)


def _matrix(t, shape, dtype, device, name):
    """A [rows, cols] tensor as (address, leading stride); (None, 0) for None."""
    if t is None:
        return _NONE
    try:
        ld, one = t.stride()
        ok = t.shape == shape and t.dtype is dtype and t.device == device and (one == 1 or shape[1] <= 1)
    except (AttributeError, ValueError):
        ok = False
    if not ok:
        _refuse(t, shape, dtype, device, name)
    return t.data_ptr(), ld if shape[0] > 1 else max(ld, shape[1])


def _vector(t, n, dtype, device, name):
    if t is None:
        return None
    if not (t.shape == (n,) and t.dtype is dtype and t.device == device and t.is_contiguous()):
        _refuse(t, (n,), dtype, device, name)
    return t.data_ptr()


def _type(t, name):
    _need(isinstance(t, _torch.Tensor) and t.is_cuda, f"{name}: want a device tensor")
    code = _types.get(t.dtype)
    if code is None:
        raise ValueError(f"{name}: {t.dtype} is not float32, float16 or bfloat16")
    return code


def _call(name, a, device, stream, used):
    """Launch on the tensors' device, with a workspace where one is needed."""
    if device.index != _torch.cuda.current_device():
        with _torch.cuda.device(device):
            return _call(name, a, device, stream, used)
    run = getattr(_lib, name)
    handle, other = _stream(stream, device)
    code = run(ctypes.byref(a), handle)
    if code == E_CAPACITY:
        need = getattr(_lib, name + "_workspace")(ctypes.byref(a))
        ws = _torch.empty(need, dtype=_torch.uint8, device=device)
        a.workspace, a.workspace_bytes = ws.data_ptr(), need
        used = (*used, ws)
        code = run(ctypes.byref(a), handle)
    if code:
        _check(code, name)
    if other is not None:
        _keep(other, used)


def _stream(stream, device):
    """(its handle, the stream itself where it is not the current one)"""
    current = _raw_stream(device.index)
    if stream is None:
        return current, None
    handle = getattr(stream, "cuda_stream", stream)
    return handle, None if handle == current else stream


def _keep(stream, tensors):
    """Memory that torch's allocator gave to the current stream and that another
    one works on is not given out again before that one has passed."""
    if not isinstance(stream, _torch.cuda.Stream):
        stream = _torch.cuda.ExternalStream(stream)
    for t in tensors:
        if t is not None:
            t.record_stream(stream)


def linear(x, w, bias=None, act="none", dropout=None, residual=None, pre=None, out=None,
           stream=None):
    """``residual + D(act(x w^T + bias))``: x [m, k], w [n, k], bias [n], residual
    and the result [m, n]; float16 or bfloat16, summed in float32.  ``pre``, if
    given, receives ``x w^T + bias``, which linear_backward needs when there is an
    activation.  A result allocated here belongs to torch's current stream."""
    _load()
    code, dt, dev = _type(x, "x"), x.dtype, x.device
    _need(x.dim() == 2 and w.dim() == 2, "x and w are matrices")
    (m, k), n = x.shape, w.shape[0]
    if out is None:
        out = _torch.empty((m, n), dtype=dt, device=dev)
    a = _Linear(m, n, k, code, _act(act), *_matrix(x, (m, k), dt, dev, "x"),
                *_matrix(w, (n, k), dt, dev, "w"), _vector(bias, n, dt, dev, "bias"),
                *_matrix(residual, (m, n), dt, dev, "residual"),
                dropout if dropout is not None else _NO_DROP,
                *_matrix(out, (m, n), dt, dev, "out"),
                *_matrix(pre, (m, n), dt, dev, "pre"), None, 0)
    _call("dip_linear", a, dev, stream, (x, w, bias, residual, pre, out))
    return out


def linear_backward(dy, x, w, act="none", dropout=None, pre=None, bias=True, need_dx=True,
                    need_dw=True, dx=None, dw=None, db=None, accumulate=False, stream=None):
    """Gradients (dx, dw, db) of linear for the gradient ``dy`` of its result;
    None for those not asked for.  ``dx``, ``dw`` and ``db`` may be given; dw and
    db may then be float32, and with ``accumulate`` they are added to.  The
    residual's gradient is dy."""
    _load()
    code, dt, dev = _type(dy, "dy"), dy.dtype, dy.device
    _need(dy.dim() == 2 and x.dim() == 2 and w.dim() == 2, "dy, x and w are matrices")
    (m, n), k = dy.shape, x.shape[1]
    _need(act == "none" or pre is not None, f"{act}: pre (the forward's) is needed")
    given = [t for t in (dw, db) if t is not None]
    _need(not accumulate or (not need_dw or dw is not None) and (not bias or db is not None),
          "accumulate: dw and db have to be given")
    gt = given[0].dtype if given else dt
    _need(all(t.dtype == gt for t in given) and gt in (dt, _torch.float32),
          "dw and db are both of dy's type or both float32")
    if need_dx and dx is None:
        dx = _torch.empty((m, k), dtype=dt, device=dev)
    if need_dw and dw is None:
        dw = _torch.empty((n, k), dtype=gt, device=dev)
    if bias and db is None:
        db = _torch.empty((n,), dtype=gt, device=dev)
    dx, dw, db = dx if need_dx else None, dw if need_dw else None, db if bias else None
    a = _LinearGrad(m, n, k, code, _act(act), *_matrix(dy, (m, n), dt, dev, "dy"),
                    *_matrix(x, (m, k), dt, dev, "x"), *_matrix(w, (n, k), dt, dev, "w"),
                    *_matrix(pre if act != "none" else None, (m, n), dt, dev, "pre"),
                    dropout if dropout is not None else _NO_DROP,
                    *_matrix(dx, (m, k), dt, dev, "dx"),
                    *_matrix(dw, (n, k), gt, dev, "dw"),
                    _vector(db, n, gt, dev, "db"), _types[gt], int(bool(accumulate)), None, 0)
    _call("dip_linear_grad", a, dev, stream, (dy, x, w, pre, dx, dw, db))
    return dx, dw, db


def dropout_add(x, dropout, residual=None, out=None, stream=None):
    """``residual + D(x)`` for x [m, n]; ``dropout_add(dy, dropout)`` is the
    gradient of x."""
    _load()
    code, dt, dev = _type(x, "x"), x.dtype, x.device
    _need(x.dim() == 2, "x is a matrix")
    m, n = x.shape
    if out is None:
        out = _torch.empty((m, n), dtype=dt, device=dev)
    px, ldx = _matrix(x, (m, n), dt, dev, "x")
    pr, ldr = _matrix(residual, (m, n), dt, dev, "residual")
    py, ldy = _matrix(out, (m, n), dt, dev, "out")
    if dev.index != _torch.cuda.current_device():
        with _torch.cuda.device(dev):
            return dropout_add(x, dropout, residual, out, stream)
    handle, other = _stream(stream, dev)
    code = _lib.dip_dropout_add(code, m, n, px, ldx, pr, ldr, ctypes.byref(dropout), py, ldy, handle)
    if code:
        _check(code, "dip_dropout_add")
    if other is not None:
        _keep(other, (x, residual, out))
    return out


def _rows(t, shape, dtype, device, name):
    """A [b, s, c] tensor as (address, sample stride, position stride)."""
    if t is None:
        return None, 0, 0
    try:
        sb, ss, one = t.stride()
        ok = t.shape == shape and t.dtype is dtype and t.device == device and (one == 1 or shape[2] <= 1)
    except (AttributeError, ValueError):
        ok = False
    if not ok:
        _refuse(t, shape, dtype, device, name)
    return t.data_ptr(), sb, ss


def group_norm(x, groups, gamma=None, beta=None, eps=1e-5, act="none", out=None, mean=None,
               rstd=None, stream=None):
    """(y, mean, rstd): group norm of x [b, s, c] (channels last) and its
    activation; float32 statistics [b, groups] for group_norm_backward.  One
    position and one group a sample make it a layer norm of the rows."""
    _load()
    code, dt, dev = _type(x, "x"), x.dtype, x.device
    _need(x.dim() == 3, "x is [samples, positions, channels]")
    b, s, c = x.shape
    out = _torch.empty((b, s, c), dtype=dt, device=dev) if out is None else out
    _need(1 <= groups < 1 << 31, f"{groups} groups")
    mean, rstd = (t if t is not None else _torch.empty((b, groups), dtype=_torch.float32, device=dev)
                  for t in (mean, rstd))
    f32 = _torch.float32
    a = _GroupNorm(b, s, c, groups, code, _act(act), eps, *_rows(x, (b, s, c), dt, dev, "x"),
                   _vector(gamma, c, dt, dev, "gamma"), _vector(beta, c, dt, dev, "beta"),
                   *_rows(out, (b, s, c), dt, dev, "out"),
                   _vector(mean.view(-1), b * groups, f32, dev, "mean"),
                   _vector(rstd.view(-1), b * groups, f32, dev, "rstd"), None, 0)
    _call("dip_group_norm", a, dev, stream, (x, gamma, beta, out, mean, rstd))
    return out, mean, rstd


def group_norm_backward(dy, x, mean, rstd, groups, gamma=None, beta=None, act="none", need_dx=True,
                        need_dparam=True, dx=None, stream=None):
    """Gradients (dx, dgamma, dbeta) of group_norm; dgamma and dbeta are None
    without ``need_dparam`` or where gamma and beta are None."""
    _load()
    code, dt, dev = _type(dy, "dy"), dy.dtype, dy.device
    _need(dy.dim() == 3, "dy is [samples, positions, channels]")
    _need(mean is not None and rstd is not None, "mean and rstd (the forward's) are needed")
    b, s, c = dy.shape
    f32 = _torch.float32
    _need(1 <= groups < 1 << 31, f"{groups} groups")
    if need_dx and dx is None:
        dx = _torch.empty((b, s, c), dtype=dt, device=dev)
    dx = dx if need_dx else None
    dgamma = _torch.empty((c,), dtype=dt, device=dev) if need_dparam and gamma is not None else None
    dbeta = _torch.empty((c,), dtype=dt, device=dev) if need_dparam and beta is not None else None
    a = _GroupNormGrad(b, s, c, groups, code, _act(act), *_rows(dy, (b, s, c), dt, dev, "dy"),
                       *_rows(x, (b, s, c), dt, dev, "x"), _vector(gamma, c, dt, dev, "gamma"),
                       _vector(beta, c, dt, dev, "beta"),
                       _vector(mean.view(-1), b * groups, f32, dev, "mean"),
                       _vector(rstd.view(-1), b * groups, f32, dev, "rstd"),
                       *_rows(dx, (b, s, c), dt, dev, "dx"),
                       dgamma.data_ptr() if dgamma is not None else None,
                       dbeta.data_ptr() if dbeta is not None else None, None, 0)
    _call("dip_group_norm_grad", a, dev, stream, (dy, x, mean, rstd, gamma, beta, dx, dgamma, dbeta))
    return dx, dgamma, dbeta

"""Python binding of the stage operators (include/dip_ops.h).

The operators that the cost tables price -- matrix product with its epilogue,
dropout whose mask is never stored, group norm (layer norm) with an activation
-- forward and their gradients, as HIP kernels of ``libdip_sim.so``.  Functions
take torch device tensors (the last dimension contiguous, rows that do not overlap),
check them, and enqueue on ``stream`` (torch's current one by default), to which
results and workspaces that a call allocates belong, as if that stream were the
current one.  As in the rest of the package PyTorch provides device memory and the
stream, nothing else: outputs and workspaces come from its allocator where none is
given, and no call records an autograd graph: a forward of tensors that require
gradients, where torch records them, warns that its result is cut off from theirs.
"""
from __future__ import annotations

import ctypes
import struct
import warnings

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
                ("act", _i32), ("accumulate", _i32), ("dy", _vp), ("dy_sb", _i64), ("dy_ss", _i64), ("x", _vp),
                ("x_sb", _i64), ("x_ss", _i64), ("gamma", _vp), ("beta", _vp), ("mean", _vp),
                ("rstd", _vp), ("dx", _vp), ("dx_sb", _i64), ("dx_ss", _i64), ("dgamma", _vp),
                ("dbeta", _vp), ("workspace", _vp), ("workspace_bytes", _i64)]


# A call's arguments go to the library as the bytes of its struct, in one step.
_CODES = {_i64: "q", _i32: "i", ctypes.c_float: "f", _vp: "Q", Dropout: "QQII"}


def _packer(cls):
    return struct.Struct("@" + "".join(_CODES[t] for _, t in cls._fields_)).pack


_pack_linear, _pack_linear_grad = _packer(_Linear), _packer(_LinearGrad)
_pack_norm, _pack_norm_grad = _packer(_GroupNorm), _packer(_GroupNormGrad)
_WORKSPACE = struct.Struct("@Qq")   # every struct's last two members

_lib = None
_torch = None
_empty = None
_raw_stream = None   # device index -> handle of torch's current stream
_device = None       # () -> index of the current device
_recording = None    # () -> whether torch records gradients
_types = {}


def _load():
    """The library with the operators' signatures, and torch."""
    global _lib, _torch, _empty, _raw_stream, _device, _recording
    if _lib is None:
        import torch
        lib = load()
        for name in ("dip_linear", "dip_linear_grad", "dip_group_norm", "dip_group_norm_grad"):
            getattr(lib, name).argtypes = [_vp, _vp]
            getattr(lib, name).restype = ctypes.c_int
            getattr(lib, name + "_workspace").argtypes = [_vp]
            getattr(lib, name + "_workspace").restype = _i64
        lib.dip_dropout_add.argtypes = [_i32, _i64, _i64, _vp, _i64, _vp, _i64,
                                        ctypes.POINTER(Dropout), _vp, _i64, _vp]
        lib.dip_dropout_add.restype = ctypes.c_int
        _types.update({torch.float32: F32, torch.float16: F16, torch.bfloat16: BF16})
        _raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream",
                              lambda index: torch.cuda.current_stream(index).cuda_stream)
        _device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)
        _recording = torch.is_grad_enabled
        _torch, _empty, _lib = torch, torch.empty, lib
    return _lib


_NO_DROP = (0, 0, 0, 0)


def _need(ok: bool, what: str):
    if not ok:
        raise ValueError(what)


def _cut_off(name):
    warnings.warn(f"{name} records no gradients: its result is cut off from tensors that require them; run its "
                  f"backward yourself, or call it without recording (torch.no_grad, detach)", stacklevel=3)


def _act(name) -> int:
    code = ACTS.get(name)
    if code is None:
        raise ValueError(f"unknown activation {name!r}: one of {', '.join(ACTS)}")
    return code


def _drop(d):
    return _NO_DROP if d is None else (d.seed, d.offset, d.row0, d.drop_of)


def _refuse(t, shape, dtype, index, name):
    if not isinstance(t, _torch.Tensor):
        raise ValueError(f"{name}: want a tensor, got {type(t).__name__}")
    if t.shape != shape or t.dtype != dtype or t.get_device() != index:
        raise ValueError(f"{name}: want {tuple(shape)} {dtype} on cuda:{index}, "
                         f"got {tuple(t.shape)} {t.dtype} on {t.device}")
    raise ValueError(f"{name}: the last dimension has to be contiguous")


_NONE, _NONE3 = (0, 0), (0, 0, 0)


def _matrix(t, shape, dtype, index, name):
    """A [rows, cols] tensor as (address, leading stride); zeros for None."""
    if t is None:
        return _NONE
    try:
        ld, one = t.stride()
        if t.shape == shape and t.dtype is dtype and t.get_device() == index and (one == 1 or shape[1] <= 1):
            return t.data_ptr(), ld if shape[0] > 1 else -(-shape[1] // 8) * 8   # one row: any
    except (AttributeError, ValueError):
        pass
    _refuse(t, shape, dtype, index, name)


def _rows(t, shape, dtype, index, name):
    """A [b, s, c] tensor as (address, sample stride, position stride)."""
    if t is None:
        return _NONE3
    try:
        sb, ss, one = t.stride()
        if t.shape == shape and t.dtype is dtype and t.get_device() == index and (one == 1 or shape[2] <= 1):
            return t.data_ptr(), sb, ss
    except (AttributeError, ValueError):
        pass
    _refuse(t, shape, dtype, index, name)


def _whole(t, shape, dtype, index, name):
    """The address of a contiguous tensor; zero for None."""
    if t is None:
        return 0
    if isinstance(t, _torch.Tensor) and t.shape == shape and t.dtype is dtype and t.get_device() == index \
            and t.is_contiguous():
        return t.data_ptr()
    _refuse(t, shape, dtype, index, name)


def _type(t, name):
    """(code, dtype, device index) of an operator's first tensor."""
    if not isinstance(t, _torch.Tensor) or not t.is_cuda:
        raise ValueError(f"{name}: want a device tensor")
    dtype = t.dtype
    code = _types.get(dtype)
    if code is None:
        raise ValueError(f"{name}: {dtype} is not float32, float16 or bfloat16")
    return code, dtype, t.get_device()


def _call(name, args, index):
    """Launch on the tensors' device and its current stream, with a workspace where
    one is needed."""
    if index != _device():
        with _torch.cuda.device(index):
            return _call(name, args, index)
    run = getattr(_lib, name)
    handle = _raw_stream(index)
    code = run(args, handle)
    if code == E_CAPACITY:
        need = getattr(_lib, name + "_workspace")(args)
        ws = _empty(need, dtype=_torch.uint8, device=_torch.device("cuda", index))
        code = run(args[:-_WORKSPACE.size] + _WORKSPACE.pack(ws.data_ptr(), need), handle)
    if code:
        _check(code, name)


def _on(stream, operator, *args):
    """operator(*args) with ``stream`` (or a handle of one) as the current stream, so
    that results and workspaces come from its pool: a block of another stream's may
    still be in use by that stream's pending work, which nothing orders before this
    call.  What was given belongs to the caller; its memory is not handed out again
    before ``stream`` has passed the call."""
    index = args[0].get_device()
    handle = getattr(stream, "cuda_stream", stream)
    if not isinstance(stream, _torch.cuda.Stream):
        stream = _torch.cuda.ExternalStream(handle, device=_torch.device("cuda", index))
    elif stream.device.index != index:
        raise ValueError(f"the stream is of {stream.device}, the tensors are on cuda:{index}")
    if handle == _raw_stream(index):
        return operator(*args)
    with _torch.cuda.stream(stream):
        out = operator(*args)
    for t in args:
        if isinstance(t, _torch.Tensor):
            t.record_stream(stream)
    return out


def linear(x, w, bias=None, act="none", dropout=None, residual=None, pre=None, out=None,
           stream=None):
    """``residual + D(act(x w^T + bias))``: x [m, k], w [n, k], bias [n], residual
    and the result [m, n]; float16 or bfloat16, summed in float32.  ``pre``, if
    given, receives ``x w^T + bias``, which linear_backward needs when there is an
    activation."""
    if _lib is None:
        _load()
    code, dt, dev = _type(x, "x")
    if stream is not None:
        return _on(stream, linear, x, w, bias, act, dropout, residual, pre, out)
    _need(x.dim() == 2 and w.dim() == 2, "x and w are matrices")
    m, k = x.shape
    n = w.shape[0]
    if out is None:
        out = x.new_empty((m, n))
    args = _pack_linear(m, n, k, code, _act(act), *_matrix(x, (m, k), dt, dev, "x"),
                        *_matrix(w, (n, k), dt, dev, "w"), _whole(bias, (n,), dt, dev, "bias"),
                        *_matrix(residual, (m, n), dt, dev, "residual"), *_drop(dropout),
                        *_matrix(out, (m, n), dt, dev, "out"), *_matrix(pre, (m, n), dt, dev, "pre"),
                        0, 0)
    if _recording() and (x.requires_grad or w.requires_grad or bias is not None and bias.requires_grad
                         or residual is not None and residual.requires_grad):
        _cut_off("linear")
    _call("dip_linear", args, dev)
    return out


def linear_backward(dy, x, w, act="none", dropout=None, pre=None, bias=True, need_dx=True,
                    need_dw=True, dx=None, dw=None, db=None, accumulate=False, stream=None):
    """Gradients (dx, dw, db) of linear for the gradient ``dy`` of its result;
    None for those not asked for.  ``dx``, ``dw`` and ``db`` may be given; dw and
    db may then be float32, and with ``accumulate`` they are added to.  The
    residual's gradient is dy."""
    if _lib is None:
        _load()
    code, dt, dev = _type(dy, "dy")
    if stream is not None:
        return _on(stream, linear_backward, dy, x, w, act, dropout, pre, bias, need_dx, need_dw, dx, dw, db,
                   accumulate)
    _need(dy.dim() == 2 and x.dim() == 2 and w.dim() == 2, "dy, x and w are matrices")
    m, n = dy.shape
    k = x.shape[1]
    _need(act == "none" or pre is not None, f"{act}: pre (the forward's) is needed")
    if accumulate:
        _need((not need_dw or dw is not None) and (not bias or db is not None),
              "accumulate: dw and db have to be given")
    gt = dw.dtype if dw is not None else db.dtype if db is not None else dt
    _need((gt is dt or gt is _torch.float32) and (db is None or db.dtype is gt),
          "dw and db are both of dy's type or both float32")
    if not need_dx:
        dx = None
    elif dx is None:
        dx = dy.new_empty((m, k))
    if not need_dw:
        dw = None
    elif dw is None:
        dw = dy.new_empty((n, k), dtype=gt)
    if not bias:
        db = None
    elif db is None:
        db = dy.new_empty((n,), dtype=gt)
    args = _pack_linear_grad(m, n, k, code, _act(act), *_matrix(dy, (m, n), dt, dev, "dy"),
                             *_matrix(x, (m, k), dt, dev, "x"), *_matrix(w, (n, k), dt, dev, "w"),
                             *_matrix(pre if act != "none" else None, (m, n), dt, dev, "pre"),
                             *_drop(dropout), *_matrix(dx, (m, k), dt, dev, "dx"),
                             *_matrix(dw, (n, k), gt, dev, "dw"), _whole(db, (n,), gt, dev, "db"),
                             _types[gt], int(bool(accumulate)), 0, 0)
    _call("dip_linear_grad", args, dev)
    return dx, dw, db


def dropout_add(x, dropout, residual=None, out=None, stream=None):
    """``residual + D(x)`` for x [m, n]; ``dropout_add(dy, dropout)`` is the
    gradient of x."""
    if _lib is None:
        _load()
    code, dt, dev = _type(x, "x")
    if stream is not None:
        return _on(stream, dropout_add, x, dropout, residual, out)
    _need(x.dim() == 2, "x is a matrix")
    shape = m, n = x.shape
    if out is None:
        out = x.new_empty(shape)
    px, ldx = _matrix(x, shape, dt, dev, "x")
    pr, ldr = _matrix(residual, shape, dt, dev, "residual")
    py, ldy = _matrix(out, shape, dt, dev, "out")
    if dev != _device():
        with _torch.cuda.device(dev):
            return dropout_add(x, dropout, residual, out)
    if _recording() and (x.requires_grad or residual is not None and residual.requires_grad):
        _cut_off("dropout_add")
    code = _lib.dip_dropout_add(code, m, n, px, ldx, pr, ldr, dropout, py, ldy, _raw_stream(dev))
    if code:
        _check(code, "dip_dropout_add")
    return out


def group_norm(x, groups, gamma=None, beta=None, eps=1e-5, act="none", out=None, mean=None,
               rstd=None, stream=None):
    """(y, mean, rstd): group norm of x [b, s, c] (channels last) and its
    activation; float32 statistics [b, groups] for group_norm_backward.  One
    position and one group a sample make it a layer norm of the rows."""
    if _lib is None:
        _load()
    code, dt, dev = _type(x, "x")
    if stream is not None:
        return _on(stream, group_norm, x, groups, gamma, beta, eps, act, out, mean, rstd)
    _need(x.dim() == 3, "x is [samples, positions, channels]")
    _need(1 <= groups < 1 << 31, f"{groups} groups")
    shape = b, s, c = x.shape
    f32, stats = _torch.float32, (b, groups)
    if out is None:
        out = x.new_empty(shape)
    if mean is None:
        mean = x.new_empty(stats, dtype=f32)
    if rstd is None:
        rstd = x.new_empty(stats, dtype=f32)
    args = _pack_norm(b, s, c, groups, code, _act(act), eps, *_rows(x, shape, dt, dev, "x"),
                      _whole(gamma, (c,), dt, dev, "gamma"), _whole(beta, (c,), dt, dev, "beta"),
                      *_rows(out, shape, dt, dev, "out"), _whole(mean, stats, f32, dev, "mean"),
                      _whole(rstd, stats, f32, dev, "rstd"), 0, 0)
    if _recording() and (x.requires_grad or gamma is not None and gamma.requires_grad
                         or beta is not None and beta.requires_grad):
        _cut_off("group_norm")
    _call("dip_group_norm", args, dev)
    return out, mean, rstd


def group_norm_backward(dy, x, mean, rstd, groups, gamma=None, beta=None, act="none", need_dx=True,
                        need_dparam=True, dx=None, stream=None, dgamma=None, dbeta=None, accumulate=False):
    """Gradients (dx, dgamma, dbeta) of group_norm; dgamma and dbeta are None
    without ``need_dparam`` or where gamma and beta are None.  They may be given; with
    ``accumulate`` they have to be, are float32 and are added to."""
    if _lib is None:
        _load()
    code, dt, dev = _type(dy, "dy")
    if stream is not None:
        return _on(stream, group_norm_backward, dy, x, mean, rstd, groups, gamma, beta, act, need_dx, need_dparam, dx, None,
                   dgamma, dbeta, accumulate)
    _need(dy.dim() == 3, "dy is [samples, positions, channels]")
    _need(1 <= groups < 1 << 31, f"{groups} groups")
    _need(mean is not None and rstd is not None, "mean and rstd (the forward's) are needed")
    shape = b, s, c = dy.shape
    f32, stats = _torch.float32, (b, groups)
    if not need_dx:
        dx = None
    elif dx is None:
        dx = dy.new_empty(shape)
    pt = dt
    if accumulate or dgamma is not None or dbeta is not None:
        pt = f32 if accumulate else dt
        _need((dgamma is None or gamma is not None) and (dbeta is None or beta is not None),
              "dgamma and dbeta go with gamma and beta")
        _need(not accumulate or not need_dparam or ((dgamma is not None or gamma is None)
                                                    and (dbeta is not None or beta is None)),
              "accumulate: dgamma and dbeta have to be given")
    pg = pb = 0
    if not need_dparam:
        dgamma = dbeta = None
    else:
        if dgamma is not None:
            pg = _whole(dgamma, (c,), pt, dev, "dgamma")
        elif gamma is not None:
            dgamma = dy.new_empty((c,))
            pg = dgamma.data_ptr()
        if dbeta is not None:
            pb = _whole(dbeta, (c,), pt, dev, "dbeta")
        elif beta is not None:
            dbeta = dy.new_empty((c,))
            pb = dbeta.data_ptr()
    args = _pack_norm_grad(b, s, c, groups, code, _act(act), int(bool(accumulate)), *_rows(dy, shape, dt, dev, "dy"),
                           *_rows(x, shape, dt, dev, "x"), _whole(gamma, (c,), dt, dev, "gamma"),
                           _whole(beta, (c,), dt, dev, "beta"), _whole(mean, stats, f32, dev, "mean"),
                           _whole(rstd, stats, f32, dev, "rstd"), *_rows(dx, shape, dt, dev, "dx"),
                           pg, pb, 0, 0)
    _call("dip_group_norm_grad", args, dev)
    return dx, dgamma, dbeta

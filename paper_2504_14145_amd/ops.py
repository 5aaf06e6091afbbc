"""Python binding of the stage operators (include/dip_ops.h).

The operators that the cost tables price -- matrix product with its epilogue,
dropout whose mask is never stored, group norm (layer norm) with an activation,
root-mean-square norm with the residual's addition, rotary positions with several
axes, activations kept in 8 bits -- forward and their gradients, as HIP kernels of
``libdip_sim.so``.  Functions
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
           "dip_group_norm_grad_workspace", "dip_group_norm_grad", "dip_pack8", "dip_unpack8",
           "dip_linear_kept_workspace", "dip_linear_kept", "dip_linear_grad_kept_workspace",
           "dip_linear_grad_kept", "dip_rms_norm", "dip_rms_norm_grad_workspace", "dip_rms_norm_grad",
           "dip_rotary")

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


class _Packed8(ctypes.Structure):
    _fields_ = [("values", _vp), ("ld", _i64), ("scales", _vp), ("lds", _i64)]


class _RmsNorm(ctypes.Structure):
    _fields_ = [("m", _i64), ("c", _i64), ("dtype", _i32), ("eps", ctypes.c_float), ("x", _vp), ("ldx", _i64),
                ("residual", _vp), ("ldr", _i64), ("gamma", _vp), ("total", _vp), ("ldt", _i64), ("y", _vp),
                ("ldy", _i64), ("packed", _Packed8), ("rstd", _vp)]


class _RmsNormGrad(ctypes.Structure):
    _fields_ = [("m", _i64), ("c", _i64), ("dtype", _i32), ("accumulate", _i32), ("dy", _vp), ("ldy", _i64),
                ("total", _vp), ("ldt", _i64), ("gamma", _vp), ("rstd", _vp), ("dtotal", _vp), ("lddt", _i64),
                ("dx", _vp), ("lddx", _i64), ("dgamma", _vp), ("workspace", _vp), ("workspace_bytes", _i64)]


class _Rotary(ctypes.Structure):
    _fields_ = [("t", _i64), ("heads", _i32), ("keys", _i32), ("dim", _i32), ("pairs", _i32), ("axes", _i32),
                ("dtype", _i32), ("pos_type", _i32), ("interleaved", _i32), ("inverse", _i32), ("q", _vp),
                ("q_st", _i64), ("q_sh", _i64), ("k", _vp), ("k_st", _i64), ("k_sh", _i64), ("pos", _vp),
                ("p_st", _i64), ("p_sa", _i64), ("freq", _vp), ("axis", _vp), ("q_out", _vp), ("qo_st", _i64),
                ("qo_sh", _i64), ("k_out", _vp), ("ko_st", _i64), ("ko_sh", _i64)]


# A call's arguments go to the library as the bytes of its struct, in one step.
_CODES = {_i64: "q", _i32: "i", ctypes.c_float: "f", _vp: "Q", Dropout: "QQII", _Packed8: "QqQq"}


def _packer(cls):
    return struct.Struct("@" + "".join(_CODES[t] for _, t in cls._fields_)).pack


_pack_linear, _pack_linear_grad = _packer(_Linear), _packer(_LinearGrad)
_pack_norm, _pack_norm_grad = _packer(_GroupNorm), _packer(_GroupNormGrad)
_pack_packed, _pack_rms, _pack_rms_grad = _packer(_Packed8), _packer(_RmsNorm), _packer(_RmsNormGrad)
_pack_rotary = _packer(_Rotary)
_WORKSPACE = struct.Struct("@Qq")   # the last two members of every struct that has a workspace

_lib = None
_torch = None
_empty = None
_raw_stream = None   # device index -> handle of torch's current stream
_device = None       # () -> index of the current device
_recording = None    # () -> whether torch records gradients
_types = {}
_positions = {}


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
        lib.dip_rms_norm_grad.argtypes = [_vp, _vp]
        lib.dip_rms_norm_grad_workspace.argtypes = [_vp]
        lib.dip_rms_norm_grad_workspace.restype = _i64
        lib.dip_rms_norm.argtypes = lib.dip_rotary.argtypes = [_vp, _vp]
        lib.dip_linear_kept.argtypes = [_vp, _vp, _vp]
        lib.dip_linear_kept_workspace.argtypes = [_vp, _vp]
        lib.dip_linear_grad_kept.argtypes = [_vp, _vp, _i32, _vp, _vp]
        lib.dip_linear_grad_kept_workspace.argtypes = [_vp, _vp, _i32, _vp]
        lib.dip_linear_kept_workspace.restype = lib.dip_linear_grad_kept_workspace.restype = _i64
        lib.dip_pack8.argtypes = [_i32, _i64, _i64, _vp, _i64, _vp, _vp]
        lib.dip_unpack8.argtypes = [_i32, _i64, _i64, _vp, _i32, _vp, _i64, _vp]
        for name in ("dip_rms_norm", "dip_rms_norm_grad", "dip_rotary", "dip_linear_kept", "dip_linear_grad_kept",
                     "dip_pack8", "dip_unpack8"):
            getattr(lib, name).restype = ctypes.c_int
        lib.dip_dropout_add.argtypes = [_i32, _i64, _i64, _vp, _i64, _vp, _i64,
                                        ctypes.POINTER(Dropout), _vp, _i64, _vp]
        lib.dip_dropout_add.restype = ctypes.c_int
        _types.update({torch.float32: F32, torch.float16: F16, torch.bfloat16: BF16})
        _positions.update({torch.int32: 0, torch.int64: 1, torch.float32: 2})
        _raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream",
                              lambda index: torch.cuda.current_stream(index).cuda_stream)
        _device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)
        _recording = torch.is_grad_enabled
        _torch, _empty, _lib = torch, torch.empty, lib
    return _lib


class Packed8:
    """A matrix [m, n] in 8 bits: ``values`` [m, n] of torch.float8_e4m3fn and a byte of
    ``scales`` [m, ceil(n / 32)] (torch.uint8) for 32 consecutive columns of a row, the
    exponent plus 127 of the power of two that their values are multiplied by.  What
    pack8 and the other operators write, and unpack8 and the gradients read."""
    __slots__ = ("values", "scales")

    def __init__(self, values, scales):
        import torch
        if not isinstance(values, torch.Tensor) or values.dim() != 2 or values.dtype is not torch.float8_e4m3fn:
            raise ValueError("values: want a matrix of float8_e4m3fn")
        shape = (values.shape[0], -(-values.shape[1] // 32))
        if not isinstance(scales, torch.Tensor) or scales.shape != shape or scales.dtype is not torch.uint8 \
                or scales.device != values.device:
            raise ValueError(f"scales: want {shape} of uint8 on {values.device}")
        self.values, self.scales = values, scales

    @classmethod
    def empty(cls, m: int, n: int, device="cuda") -> "Packed8":
        if _torch is None:
            _load()
        p = cls.__new__(cls)
        p.values = _empty((m, n), dtype=_torch.float8_e4m3fn, device=device)
        p.scales = _empty((m, -(-n // 32)), dtype=_torch.uint8, device=device)
        return p

    @classmethod
    def _of(cls, x) -> "Packed8":
        """Room for the device matrix x."""
        m, n = x.shape
        p = cls.__new__(cls)
        p.values = _torch.empty_like(x, dtype=_torch.float8_e4m3fn) if x.is_contiguous() else \
            x.new_empty((m, n), dtype=_torch.float8_e4m3fn)
        p.scales = x.new_empty((m, -(-n // 32)), dtype=_torch.uint8)
        return p

    @property
    def shape(self):
        return self.values.shape

    @property
    def device(self):
        return self.values.device

    def get_device(self) -> int:
        return self.values.get_device()


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


_NONE4 = (0, 0, 0, 0)


def _like(t):
    """A contiguous tensor of t's shape and type."""
    return _torch.empty_like(t) if t.is_contiguous() else t.new_empty(t.shape)


def _packed(p, shape, index, name):
    """A Packed8 as (values, leading stride, scales, leading stride); zeros for None."""
    if p is None:
        return _NONE4
    if not isinstance(p, Packed8):
        raise ValueError(f"{name}: want a Packed8, got {type(p).__name__}")
    m, n = shape
    return (*_matrix(p.values, shape, _torch.float8_e4m3fn, index, name),
            *_matrix(p.scales, (m, -(-n // 32)), _torch.uint8, index, name + "'s scales"))


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


def _call(name, args, index, *more):
    """Launch on the tensors' device and its current stream, with a workspace where
    one is needed; ``more``: arguments after the struct."""
    if index != _device():
        with _torch.cuda.device(index):
            return _call(name, args, index, *more)
    run = getattr(_lib, name)
    handle = _raw_stream(index)
    code = run(args, *more, handle)
    if code == E_CAPACITY:
        need = getattr(_lib, name + "_workspace")(args, *more)
        ws = _empty(need, dtype=_torch.uint8, device=_torch.device("cuda", index))
        code = run(args[:-_WORKSPACE.size] + _WORKSPACE.pack(ws.data_ptr(), need), *more, handle)
    if code:
        _check(code, name)


def _call_flat(name, index, *args):
    """The same for an entry point without a struct or a workspace."""
    if index != _device():
        with _torch.cuda.device(index):
            return _call_flat(name, index, *args)
    code = getattr(_lib, name)(*args, _raw_stream(index))
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
        elif isinstance(t, Packed8):
            t.values.record_stream(stream)
            t.scales.record_stream(stream)
    return out


def linear(x, w, bias=None, act="none", dropout=None, residual=None, pre=None, out=None,
           stream=None):
    """``residual + D(act(x w^T + bias))``: x [m, k], w [n, k], bias [n], residual
    and the result [m, n]; float16 or bfloat16, summed in float32.  ``pre``, if
    given, receives ``x w^T + bias``, which linear_backward needs when there is an
    activation; a Packed8 keeps it in 8 bits."""
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
    kept = isinstance(pre, Packed8)
    args = _pack_linear(m, n, k, code, _act(act), *_matrix(x, (m, k), dt, dev, "x"),
                        *_matrix(w, (n, k), dt, dev, "w"), _whole(bias, (n,), dt, dev, "bias"),
                        *_matrix(residual, (m, n), dt, dev, "residual"), *_drop(dropout),
                        *_matrix(out, (m, n), dt, dev, "out"),
                        *(_NONE if kept else _matrix(pre, (m, n), dt, dev, "pre")), 0, 0)
    if _recording() and (x.requires_grad or w.requires_grad or bias is not None and bias.requires_grad
                         or residual is not None and residual.requires_grad):
        _cut_off("linear")
    if kept:
        _call("dip_linear_kept", args, dev, _pack_packed(*_packed(pre, (m, n), dev, "pre")))
    else:
        _call("dip_linear", args, dev)
    return out


def linear_backward(dy, x, w, act="none", dropout=None, pre=None, bias=True, need_dx=True,
                    need_dw=True, dx=None, dw=None, db=None, accumulate=False, stream=None, x_act="none"):
    """Gradients (dx, dw, db) of linear for the gradient ``dy`` of its result;
    None for those not asked for.  ``dx``, ``dw`` and ``db`` may be given; dw and
    db may then be float32, and with ``accumulate`` they are added to.  The
    residual's gradient is dy.  ``x`` and ``pre`` may be Packed8, kept in 8 bits; such an
    x is taken through ``x_act``, the activation behind which the forward's x lay."""
    if _lib is None:
        _load()
    code, dt, dev = _type(dy, "dy")
    if stream is not None:
        return _on(stream, linear_backward, dy, x, w, act, dropout, pre, bias, need_dx, need_dw, dx, dw, db,
                   accumulate, None, x_act)
    x8, pre8 = isinstance(x, Packed8), isinstance(pre, Packed8)
    _need(dy.dim() == 2 and (x8 or x.dim() == 2) and w.dim() == 2, "dy, x and w are matrices")
    _need(x8 or x_act == "none", "x_act goes with an x kept in 8 bits")
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
                             *(_NONE if x8 else _matrix(x, (m, k), dt, dev, "x")),
                             *_matrix(w, (n, k), dt, dev, "w"),
                             *_matrix(pre if act != "none" and not pre8 else None, (m, n), dt, dev, "pre"),
                             *_drop(dropout), *_matrix(dx, (m, k), dt, dev, "dx"),
                             *_matrix(dw, (n, k), gt, dev, "dw"), _whole(db, (n,), gt, dev, "db"),
                             _types[gt], int(bool(accumulate)), 0, 0)
    if x8 or pre8:
        _call("dip_linear_grad_kept", args, dev, _pack_packed(*_packed(x, (m, k), dev, "x")) if x8 else None,
              _act(x_act), _pack_packed(*_packed(pre, (m, n), dev, "pre")) if pre8 else None)
    else:
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


def pack8(x, out=None, stream=None):
    """A matrix x [m, n] of float32, float16 or bfloat16 in 8 bits (Packed8): 32
    consecutive columns of a row share the smallest power of two by which the largest
    of them divides to at most 448, and are rounded to nearest even with four
    significant bits.  Infinities become NaN."""
    if _lib is None:
        _load()
    code, dt, dev = _type(x, "x")
    if stream is not None:
        return _on(stream, pack8, x, out)
    _need(x.dim() == 2, "x is a matrix")
    shape = m, n = x.shape
    if out is None:
        out = Packed8._of(x)
        args = _pack_packed(out.values.data_ptr(), n, out.scales.data_ptr(), -(-n // 32))
    else:
        args = _pack_packed(*_packed(out, shape, dev, "out"))
    px, ldx = _matrix(x, shape, dt, dev, "x")
    if _recording() and x.requires_grad:
        _cut_off("pack8")
    _call_flat("dip_pack8", dev, code, m, n, px, ldx, args)
    return out


def unpack8(p, dtype=None, act="none", out=None, stream=None):
    """``act`` of the matrix in 8 bits ``p``, of type ``dtype`` (bfloat16, or that of
    ``out``); without an activation exact, but for what rounded up beyond the type's
    largest value and becomes that."""
    if _lib is None:
        _load()
    _need(isinstance(p, Packed8), "p: want a Packed8")
    _need(p.values.is_cuda, "p: want device tensors")
    dev = p.get_device()
    if stream is not None:
        return _on(stream, unpack8, p, dtype, act, out)
    if dtype is None:
        dtype = _torch.bfloat16 if out is None else out.dtype
    code = _types.get(dtype)
    _need(code is not None, f"{dtype} is not float32, float16 or bfloat16")
    shape = m, n = p.shape
    args = _pack_packed(*_packed(p, shape, dev, "p"))
    if out is None:
        out = p.values.new_empty(shape, dtype=dtype)
        py, ldy = out.data_ptr(), n
    else:
        py, ldy = _matrix(out, shape, dtype, dev, "out")
    _call_flat("dip_unpack8", dev, code, m, n, args, _act(act), py, ldy)
    return out


def rms_norm(x, gamma=None, eps=1e-5, residual=None, packed=None, need_out=True, out=None, total=None, rstd=None,
             stream=None):
    """(y, total, rstd, packed): ``total = x + residual`` rounded to the type (x itself
    without a residual) and its root-mean-square norm ``y = gamma total rstd``, for x
    [m, c].  total and the float32 rstd [m] are what rms_norm_backward needs.
    ``packed``: True, or a Packed8 to fill, for y in 8 bits (what linear_backward takes
    as the x of the product that follows); y is None without ``need_out``.  ``total``
    may be the residual itself."""
    if _lib is None:
        _load()
    code, dt, dev = _type(x, "x")
    if stream is not None:
        return _on(stream, rms_norm, x, gamma, eps, residual, packed, need_out, out, total, rstd)
    _need(x.dim() == 2, "x is a matrix")
    shape = m, c = x.shape
    py = pt = _NONE
    pp = _NONE4
    # what is allocated here needs no check
    if not need_out:
        out = None
    elif out is None:
        out = _like(x)
        py = out.data_ptr(), c
    else:
        py = _matrix(out, shape, dt, dev, "out")
    if residual is None:
        _need(total is None, "total goes with a residual: without one it is x")
    elif total is None:
        total = _like(x)
        pt = total.data_ptr(), c
    else:
        pt = _matrix(total, shape, dt, dev, "total")
    if rstd is None:
        rstd = x.new_empty((m,), dtype=_torch.float32)
        pr = rstd.data_ptr()
    else:
        pr = _whole(rstd, (m,), _torch.float32, dev, "rstd")
    if packed is True:
        packed = Packed8._of(x)
        pp = packed.values.data_ptr(), c, packed.scales.data_ptr(), -(-c // 32)
    elif packed is False:
        packed = None
    else:
        pp = _packed(packed, shape, dev, "packed")
    args = _pack_rms(m, c, code, eps, *_matrix(x, shape, dt, dev, "x"), *_matrix(residual, shape, dt, dev, "residual"),
                     _whole(gamma, (c,), dt, dev, "gamma"), *pt, *py, *pp, pr)
    if _recording() and (x.requires_grad or gamma is not None and gamma.requires_grad
                         or residual is not None and residual.requires_grad):
        _cut_off("rms_norm")
    _call("dip_rms_norm", args, dev)
    return out, x if residual is None else total, rstd, packed


def rms_norm_backward(dy, total, rstd, gamma=None, dtotal=None, need_dx=True, need_dgamma=True, dx=None, dgamma=None,
                      accumulate=False, stream=None):
    """Gradients (dx, dgamma) of rms_norm for those of y and, ``dtotal``, of total: dx
    is the gradient of x and of the residual.  dgamma is None without ``need_dgamma`` or
    gamma.  dx may be dtotal itself; with ``accumulate`` dgamma has to be given, is
    float32 and added to."""
    if _lib is None:
        _load()
    code, dt, dev = _type(dy, "dy")
    if stream is not None:
        return _on(stream, rms_norm_backward, dy, total, rstd, gamma, dtotal, need_dx, need_dgamma, dx, dgamma, accumulate)
    _need(dy.dim() == 2, "dy is a matrix")
    _need(total is not None and rstd is not None, "total and rstd (the forward's) are needed")
    shape = m, c = dy.shape
    _need(dgamma is None or gamma is not None, "dgamma goes with gamma")
    f32 = _torch.float32
    px, pg = _NONE, 0
    if gamma is None or not need_dgamma:
        dgamma = None
    elif dgamma is None:
        _need(not accumulate, "accumulate: dgamma has to be given")
        dgamma = dy.new_empty((c,))
        pg = dgamma.data_ptr()
    else:
        pg = _whole(dgamma, (c,), f32 if accumulate else dt, dev, "dgamma")
    if not need_dx:
        dx = None
    elif dx is None:
        dx = _like(dy)
        px = dx.data_ptr(), c
    else:
        px = _matrix(dx, shape, dt, dev, "dx")
    args = _pack_rms_grad(m, c, code, int(bool(accumulate)), *_matrix(dy, shape, dt, dev, "dy"),
                          *_matrix(total, shape, dt, dev, "total"), _whole(gamma, (c,), dt, dev, "gamma"),
                          _whole(rstd, (m,), f32, dev, "rstd"), *_matrix(dtotal, shape, dt, dev, "dtotal"),
                          *px, pg, 0, 0)
    _call("dip_rms_norm_grad", args, dev)
    return dx, dgamma


def rotary_frequencies(sections, base=10000.0, shared=False, device="cuda"):
    """(frequencies, axis) for rotary: ``sections`` [axes] pairs of a head turn with each
    axis, in their order.  Frequencies in radians a position (float64) are base^(-i / n)
    of the i-th of an axis' n pairs or, ``shared``, of all n pairs."""
    import torch
    _need(all(isinstance(n, int) and n >= 0 for n in sections), "sections: pairs of each axis")
    pairs = sum(sections)
    freq, axis = [], []
    for a, n in enumerate(sections):
        for i in range(n):
            freq.append(float(base) ** -(len(freq) / pairs if shared else i / n))
            axis.append(a)
    return (torch.tensor(freq, dtype=torch.float64, device=device),
            torch.tensor(axis, dtype=torch.int32, device=device))


def _heads(t, tokens, dim, dtype, index, name):
    """A [tokens, heads, dim] tensor as (heads, address, token stride, head stride)."""
    if not isinstance(t, _torch.Tensor) or t.dim() != 3:
        raise ValueError(f"{name}: want a tensor [tokens, heads, elements]")
    heads = t.shape[1]
    return (heads, *_rows(t, (tokens, heads, dim), dtype, index, name))


def _turn(name, q, positions, frequencies, axis, k, interleaved, out, out_k, inverse, names):
    code, dt, dev = _type(q, names[0])
    _need(q.dim() == 3, f"{names[0]} is [tokens, heads, elements]")
    t, _, dim = q.shape
    heads, *pq = _heads(q, t, dim, dt, dev, names[0])
    keys, pk = 0, _NONE3
    if k is not None:
        keys, *pk = _heads(k, t, dim, dt, dev, names[1])
    _need(isinstance(positions, _torch.Tensor) and positions.dtype in _positions and positions.get_device() == dev,
          f"positions: want int32, int64 or float32 on cuda:{dev}")
    _need(positions.dim() in (1, 2) and positions.shape[0] == t, f"positions: want [{t}] or [{t}, axes]")
    axes, sa = (1, 0) if positions.dim() == 1 else (positions.shape[1], positions.stride(1))
    _need(isinstance(frequencies, _torch.Tensor) and frequencies.dim() == 1, "frequencies: want a tensor [pairs]")
    pairs = frequencies.shape[0]
    _need(2 * pairs <= dim, f"{pairs} pairs in a head of {dim} elements")
    po, pk_out = _NONE3, _NONE3
    if out is None:
        out = q.new_empty(q.shape)
        po = out.data_ptr(), heads * dim, dim
    else:
        po = _rows(out, q.shape, dt, dev, "out")
    if k is None:
        _need(out_k is None, "out_k goes with k")
    elif out_k is None:
        out_k = k.new_empty(k.shape)
        pk_out = out_k.data_ptr(), keys * dim, dim
    else:
        pk_out = _rows(out_k, k.shape, dt, dev, "out_k")
    args = _pack_rotary(t, heads, keys, dim, pairs, axes, code, _positions[positions.dtype], int(bool(interleaved)),
                        inverse, *pq, *pk, positions.data_ptr(), positions.stride(0), sa,
                        _whole(frequencies, (pairs,), _torch.float64, dev, "frequencies"),
                        _whole(axis, (pairs,), _torch.int32, dev, "axis"), *po, *pk_out)
    if not inverse and _recording() and (q.requires_grad or k is not None and k.requires_grad or positions.requires_grad
                                         or frequencies.requires_grad):
        _cut_off(name)
    _call("dip_rotary", args, dev)
    return out if k is None else (out, out_k)


def rotary(q, positions, frequencies, axis, k=None, interleaved=False, out=None, out_k=None, stream=None):
    """q [tokens, heads, elements] (and k, with heads of its own) turned by the tokens'
    ``positions`` [tokens, axes]: pair j of every head by ``positions[:, axis[j]]
    frequencies[j]`` radians (rotary_frequencies).  Pair j is elements j and pairs + j,
    or ``interleaved`` 2 j and 2 j + 1; elements behind the pairs are copied.  Positions
    are int32, int64 or float32; angles are float64.  A pair whose axis positions do not
    have stays as it is.  q and k may be views of one array in any order of tokens and
    heads; ``out`` may be q and ``out_k`` k themselves.  Returns q's, or both."""
    if _lib is None:
        _load()
    if stream is not None:
        _type(q, "q")
        return _on(stream, rotary, q, positions, frequencies, axis, k, interleaved, out, out_k)
    return _turn("rotary", q, positions, frequencies, axis, k, interleaved, out, out_k, 0, ("q", "k"))


def rotary_backward(dq, positions, frequencies, axis, dk=None, interleaved=False, out=None, out_k=None, stream=None):
    """The gradient of rotary's q (and k) for those of its results: the same pairs
    turned back."""
    if _lib is None:
        _load()
    if stream is not None:
        _type(dq, "dq")
        return _on(stream, rotary_backward, dq, positions, frequencies, axis, dk, interleaved, out, out_k)
    return _turn("rotary_backward", dq, positions, frequencies, axis, dk, interleaved, out, out_k, 1, ("dq", "dk"))

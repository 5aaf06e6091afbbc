"""Norm, rotary positions and 8-bit values on the CPU: struct layouts, and argument
checks, which come before any device call."""
import ctypes
import os
import re

import pytest

import paper_2504_14145_amd as dip
from paper_2504_14145_amd import ops

HEADER = os.path.join(os.path.dirname(os.path.dirname(__file__)), "include", "dip_ops.h")
AT = 1 << 20     # an address that is never read: every call here is refused or empty


@pytest.fixture(scope="module")
def lib():
    return ops._load()


def text():
    return re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)


def test_structs_and_constants_match_the_header():
    size = {"p": 8, "int64_t": 8, "int32_t": 4, "float": 4, "dip_packed8": 32}
    for cls, name in ((ops._Packed8, "dip_packed8"), (ops._RmsNorm, "dip_rms_norm_args"),
                      (ops._RmsNormGrad, "dip_rms_norm_grad_args"), (ops._Rotary, "dip_rotary_args")):
        body = re.search(r"typedef struct \{([^}]*)\} %s;" % name, text()).group(1)
        fields = []
        for line in filter(None, (v.strip() for v in body.split(";"))):
            kind = "p" if "*" in line else line.split()[0]
            for part in re.sub(r"^(const\s+)?\w+\s*", "", line).split(","):
                fields.append((part.replace("*", "").strip(), kind))
        assert [(f, size[k]) for f, k in fields] == [(n, ctypes.sizeof(t)) for n, t in cls._fields_], name
    for cls, pack in ((ops._RmsNorm, ops._pack_rms), (ops._RmsNormGrad, ops._pack_rms_grad),
                      (ops._Rotary, ops._pack_rotary), (ops._Packed8, ops._pack_packed)):
        assert pack.__self__.size == ctypes.sizeof(cls)
    const = dict(re.findall(r"#define (DIP_POS_\w+) (\d+)", text()))
    assert const == {"DIP_POS_I32": "0", "DIP_POS_I64": "1", "DIP_POS_F32": "2"}


def packed(m=4, n=40, **kw):
    p = ops._Packed8(values=AT + 3, ld=n, scales=AT + 1, lds=(n + 31) // 32)
    for k, v in kw.items():
        setattr(p, k, v)
    return p


BAD_PACKED = [(dict(values=None), dip.E_INVAL), (dict(scales=None), dip.E_INVAL), (dict(ld=39), dip.E_INVAL),
              (dict(lds=1), dip.E_INVAL), (dict(ld=(1 << 22) + 1), dip.E_RANGE)]


@pytest.mark.parametrize("change,code", BAD_PACKED)
def test_packed_refusals(lib, change, code):
    p = packed(**change)
    r = ctypes.byref(p)
    assert lib.dip_pack8(ops.BF16, 4, 40, AT, 40, r, None) == code
    assert lib.dip_unpack8(ops.BF16, 4, 40, r, 0, AT, 40, None) == code
    a = ops._Linear(m=4, n=40, k=16, dtype=ops.BF16, act=2, x=AT, ldx=16, w=AT, ldw=16, y=AT, ldy=40)
    assert lib.dip_linear_kept(ctypes.byref(a), r, None) == code
    assert lib.dip_linear_kept_workspace(ctypes.byref(a), r) == code
    g = grad()
    assert lib.dip_linear_grad_kept(ctypes.byref(g), None, 0, r, None) == code
    assert lib.dip_linear_grad_kept(ctypes.byref(g), r, 0, ctypes.byref(packed()), None) == code
    assert lib.dip_linear_grad_kept_workspace(ctypes.byref(g), r, 0, None) == code
    n = rms(packed=p)
    assert lib.dip_rms_norm(ctypes.byref(n), None) == code


def grad(**kw):
    a = ops._LinearGrad(m=4, n=40, k=40, dtype=ops.BF16, act=2, dy=AT, ldy=40, x=AT, ldx=40, w=AT, ldw=40, pre=AT, ldp=40,
                        dx=AT, lddx=40, dw=AT, lddw=40, db=AT, grad_dtype=ops.BF16, workspace=AT, workspace_bytes=1 << 24)
    for k, v in kw.items():
        setattr(a, k, v)
    return a


@pytest.mark.parametrize("change,x,x_act,pre,code", [
    (dict(dtype=ops.F32), True, 0, True, dip.E_UNSUPPORTED), ({}, True, 4, True, dip.E_INVAL),
    ({}, True, -1, True, dip.E_INVAL), (dict(pre=None), True, 0, False, dip.E_INVAL),
    (dict(x=None), False, 0, True, dip.E_INVAL), (dict(workspace_bytes=64), True, 0, True, dip.E_CAPACITY),
    (dict(workspace=AT + 8), True, 0, True, dip.E_INVAL), (dict(lddw=39), True, 0, True, dip.E_INVAL)])
def test_kept_gradient_refusals(lib, change, x, x_act, pre, code):
    a = grad(**change)
    p = packed()
    r = ctypes.byref(p)
    assert lib.dip_linear_grad_kept(ctypes.byref(a), r if x else None, x_act, r if pre else None, None) == code


def test_kept_arrays_take_the_place_of_x_and_pre(lib):
    a, p = grad(x=None, pre=None, ldx=0, ldp=0), packed()
    r = ctypes.byref(p)
    assert lib.dip_linear_grad_kept_workspace(ctypes.byref(a), r, 0, r) > 4 * 40 * 2
    assert lib.dip_linear_grad_workspace(ctypes.byref(a)) == dip.E_INVAL
    b = ops._Linear(m=4, n=40, k=16, dtype=ops.F16, x=AT, ldx=16, w=AT, ldw=16, y=AT, ldy=40, pre=AT + 1, ldp=1)
    assert lib.dip_linear_kept_workspace(ctypes.byref(b), r) >= 0          # its own pre is not used
    assert lib.dip_linear_kept(ctypes.byref(b), None, None) == dip.E_INVAL
    assert lib.dip_linear_kept(None, r, None) == dip.E_INVAL and lib.dip_linear_grad_kept(None, r, 0, r, None) == dip.E_INVAL


@pytest.mark.parametrize("change,code", [
    (dict(dtype=5), dip.E_INVAL), (dict(m=-1), dip.E_INVAL), (dict(x=None), dip.E_INVAL), (dict(x=AT + 1), dip.E_INVAL),
    (dict(ldx=39), dip.E_INVAL), (dict(m=1 << 31), dip.E_RANGE), (dict(n=1 << 23, ldx=1 << 23), dip.E_RANGE)])
def test_pack_refusals(lib, change, code):
    a = dict(dtype=ops.F16, m=4, n=40, x=AT, ldx=40) | change
    p = packed()
    assert lib.dip_pack8(a["dtype"], a["m"], a["n"], a["x"], a["ldx"], ctypes.byref(p), None) == code
    assert lib.dip_unpack8(a["dtype"], a["m"], a["n"], ctypes.byref(p), 0, a["x"], a["ldx"], None) in (code, dip.E_INVAL)
    assert lib.dip_pack8(ops.F16, 4, 40, AT, 40, None, None) == dip.E_INVAL
    assert lib.dip_unpack8(ops.F16, 4, 40, ctypes.byref(p), 7, AT, 40, None) == dip.E_INVAL


def rms(**kw):
    a = ops._RmsNorm(m=4, c=40, dtype=ops.BF16, eps=1e-5, x=AT, ldx=40, residual=AT, ldr=40, gamma=AT, total=AT, ldt=40,
                     y=AT, ldy=40, rstd=AT)
    for k, v in kw.items():
        setattr(a, k, v)
    return a


@pytest.mark.parametrize("change,code", [
    (dict(dtype=-1), dip.E_INVAL), (dict(eps=-1.0), dip.E_INVAL), (dict(eps=float("nan")), dip.E_INVAL),
    (dict(x=None), dip.E_INVAL), (dict(ldr=39), dip.E_INVAL), (dict(total=AT + 1), dip.E_INVAL), (dict(ldy=1), dip.E_INVAL),
    (dict(gamma=AT + 1), dip.E_INVAL), (dict(rstd=AT + 2), dip.E_INVAL), (dict(m=-1), dip.E_INVAL),
    (dict(m=1 << 31), dip.E_RANGE), (dict(ldx=(1 << 22) + 2), dip.E_RANGE)])
def test_norm_refusals(lib, change, code):
    assert lib.dip_rms_norm(ctypes.byref(rms(**change)), None) == code


@pytest.mark.parametrize("change,code", [
    (dict(dy=None), dip.E_INVAL), (dict(total=None), dip.E_INVAL), (dict(rstd=None), dip.E_INVAL), (dict(ldt=39), dip.E_INVAL),
    (dict(lddx=39), dip.E_INVAL), (dict(lddt=39), dip.E_INVAL), (dict(dgamma=AT + 1), dip.E_INVAL),
    (dict(dgamma=AT + 2, accumulate=1), dip.E_INVAL), (dict(workspace_bytes=0), dip.E_CAPACITY),
    (dict(workspace=AT + 8), dip.E_INVAL), (dict(dtype=3), dip.E_INVAL), (dict(m=1 << 31), dip.E_RANGE)])
def test_norm_gradient_refusals(lib, change, code):
    # more rows than those whose gradient needs no workspace
    a = ops._RmsNormGrad(m=1000, c=40, dtype=ops.BF16, dy=AT, ldy=40, total=AT, ldt=40, gamma=AT, rstd=AT, dtotal=AT, lddt=40,
                         dx=AT, lddx=40, dgamma=AT, workspace=AT, workspace_bytes=1 << 24)
    for k, v in change.items():
        setattr(a, k, v)
    assert lib.dip_rms_norm_grad(ctypes.byref(a), None) == code


@pytest.mark.parametrize("change,code", [
    (dict(dtype=3), dip.E_INVAL), (dict(pos_type=3), dip.E_INVAL), (dict(pos_type=-1), dip.E_INVAL), (dict(t=-1), dip.E_INVAL),
    (dict(pairs=21), dip.E_INVAL), (dict(pairs=-1), dip.E_INVAL), (dict(axes=-1), dip.E_INVAL), (dict(heads=-1), dip.E_INVAL),
    (dict(q=None), dip.E_INVAL), (dict(k=AT + 1), dip.E_INVAL), (dict(q_sh=39), dip.E_INVAL), (dict(q_st=159), dip.E_INVAL),
    (dict(qo_st=100), dip.E_INVAL), (dict(ko_sh=0), dip.E_INVAL), (dict(freq=None), dip.E_INVAL), (dict(freq=AT + 4), dip.E_INVAL),
    (dict(axis=AT + 2), dip.E_INVAL), (dict(pos=None), dip.E_INVAL), (dict(pos=AT + 4, pos_type=1), dip.E_INVAL),
    (dict(t=1 << 31), dip.E_RANGE), (dict(dim=2050, q_sh=4096), dip.E_RANGE), (dict(keys=1 << 20), dip.E_RANGE),
    (dict(p_st=-(1 << 50)), dip.E_RANGE), (dict(q_st=1 << 50), dip.E_RANGE)])
def test_rotary_refusals(lib, change, code):
    a = ops._Rotary(t=3, heads=4, keys=2, dim=40, pairs=20, axes=2, dtype=ops.F16, q=AT, q_st=160, q_sh=40, k=AT, k_st=80,
                    k_sh=40, pos=AT, p_st=2, p_sa=1, freq=AT, axis=AT, q_out=AT, qo_st=160, qo_sh=40, k_out=AT, ko_st=80, ko_sh=40)
    for k, v in change.items():
        setattr(a, k, v)
    assert lib.dip_rotary(ctypes.byref(a), None) == code


def test_empty_calls_are_done(lib):
    p = ops._Packed8()
    r = ctypes.byref(p)
    assert lib.dip_pack8(ops.F32, 0, 5, None, 0, r, None) == lib.dip_unpack8(ops.F32, 5, 0, r, 0, None, 0, None) == dip.OK
    assert lib.dip_rms_norm(ctypes.byref(ops._RmsNorm(m=0, c=5)), None) == dip.OK
    assert lib.dip_rms_norm_grad(ctypes.byref(ops._RmsNormGrad(m=5, c=0, dx=AT, lddx=0)), None) == dip.OK
    assert lib.dip_rotary(ctypes.byref(ops._Rotary(t=0, heads=4, dim=8, pairs=4)), None) == dip.OK
    assert lib.dip_rotary(ctypes.byref(ops._Rotary(t=5, heads=0, keys=0, dim=8, pairs=4)), None) == dip.OK
    for f in (lib.dip_rms_norm, lib.dip_rms_norm_grad, lib.dip_rotary):
        assert f(None, None) == dip.E_INVAL


def test_binding_refuses_what_is_not_on_a_device_or_of_the_kind():
    torch = pytest.importorskip("torch")
    x = torch.zeros((4, 40))
    for call in (lambda: ops.rms_norm(x), lambda: ops.rms_norm_backward(x, x, x), lambda: ops.pack8(x),
                 lambda: ops.unpack8(ops.Packed8.empty(4, 40, "cpu")), lambda: ops.unpack8(x),
                 lambda: ops.rotary(x, x, x, x), lambda: ops.rotary_backward(x, x, x, x),
                 lambda: ops.Packed8(x, x), lambda: ops.Packed8(x.to(torch.float8_e4m3fn), x),
                 lambda: ops.Packed8(x.to(torch.float8_e4m3fn), torch.zeros((4, 1), dtype=torch.uint8)),
                 lambda: ops.rotary_frequencies((4, -1), device="cpu")):
        with pytest.raises(ValueError):
            call()


def test_frequencies():
    f, a = ops.rotary_frequencies((2, 1, 0, 3), base=100.0, device="cpu")
    assert a.tolist() == [0, 0, 1, 3, 3, 3]
    assert f.tolist() == pytest.approx([1, 0.1, 1, 1, 100 ** (-1 / 3), 100 ** (-2 / 3)], rel=1e-15)
    f, _ = ops.rotary_frequencies((1, 3), base=16.0, shared=True, device="cpu")
    assert f.tolist() == pytest.approx([1, 0.5, 0.25, 0.125], rel=1e-15)
    assert ops.rotary_frequencies((), device="cpu")[0].shape == (0,)

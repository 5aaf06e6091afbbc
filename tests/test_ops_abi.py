"""The stage operators' C ABI on the CPU: declared symbols, struct layouts, and
argument checks, which come before any device call."""
import ctypes
import os
import re

import pytest

import paper_2504_14145_amd as dip
from paper_2504_14145_amd import ops

from ops_reference import philox

HEADER = os.path.join(os.path.dirname(os.path.dirname(__file__)), "include", "dip_ops.h")
AT = 1 << 20     # an address that is never read: every call here is refused or empty


@pytest.fixture(scope="module")
def lib():
    return ops._load()


def text():
    return re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)


def test_library_exports_every_declared_symbol(lib):
    names = set(re.findall(r"\b(dip_\w+)\s*\(", text()))
    assert names == set(ops.EXPORTS)
    assert all(hasattr(lib, n) for n in names)


def test_structs_and_constants_match_the_header():
    for cls, name in ((ops.Dropout, "dip_dropout"), (ops._Linear, "dip_linear_args"),
                      (ops._LinearGrad, "dip_linear_grad_args"), (ops._GroupNorm, "dip_group_norm_args"),
                      (ops._GroupNormGrad, "dip_group_norm_grad_args")):
        body = re.search(r"typedef struct \{([^}]*)\} %s;" % name, text()).group(1)
        fields = []
        for line in body.split(";"):
            line = line.strip()
            if not line:
                continue
            kind = "p" if "*" in line else line.split()[0]
            for part in re.sub(r"^(const\s+)?\w+\s*", "", line).split(","):
                fields.append((part.replace("*", "").strip(), kind))
        size = {"p": 8, "int64_t": 8, "uint64_t": 8, "int32_t": 4, "uint32_t": 4, "float": 4, "dip_dropout": 24}
        assert [(f, size[k]) for f, k in fields] == \
            [(n.lstrip("_"), ctypes.sizeof(t)) for n, t in cls._fields_], name
    const = dict(re.findall(r"#define (DIP_\w+) (\d+)", text()))
    assert [int(const[k]) for k in ("DIP_F32", "DIP_F16", "DIP_BF16")] == [ops.F32, ops.F16, ops.BF16]
    assert ops.ACTS == {k[8:].lower(): int(v) for k, v in const.items() if k.startswith("DIP_ACT_")}


def test_generator_against_published_outputs():
    """The known answers of Philox4x32-10 for counters and keys of all zeros, all
    ones, and digits of pi (Salmon et al., the generator's published tests)."""
    ones = 0xFFFFFFFF
    assert philox((0, 0, 0, 0), (0, 0)) == [0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8]
    assert philox((ones,) * 4, (ones,) * 2) == [0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD]
    assert philox((0x243F6A88, 0x85A308D3, 0x13198A2E, 0x03707344), (0xA4093822, 0x299F31D0)) == \
        [0xD16CFE09, 0x94FDCCEB, 0x5001E420, 0x24126EA1]


def linear(**kw):
    a = ops._Linear(m=4, n=8, k=16, dtype=ops.BF16, x=AT, ldx=16, w=AT, ldw=16, y=AT, ldy=8)
    for k, v in kw.items():
        setattr(a, k, v)
    return a


@pytest.mark.parametrize("change,code", [
    (dict(m=-1), dip.E_INVAL), (dict(dtype=3), dip.E_INVAL), (dict(dtype=ops.F32), dip.E_UNSUPPORTED),
    (dict(act=4), dip.E_INVAL), (dict(act=-1), dip.E_INVAL), (dict(x=None), dip.E_INVAL),
    (dict(w=AT + 1), dip.E_INVAL), (dict(y=None), dip.E_INVAL), (dict(ldx=15), dip.E_INVAL),
    (dict(ldy=7), dip.E_INVAL), (dict(residual=AT, ldr=3), dip.E_INVAL), (dict(pre=AT, ldp=0), dip.E_INVAL),
    (dict(bias=AT + 1), dip.E_INVAL), (dict(m=1 << 31), dip.E_RANGE), (dict(k=1 << 25, ldx=1 << 25, ldw=1 << 25), dip.E_RANGE),
    (dict(ldx=(1 << 24) + 1), dip.E_RANGE), (dict(drop=ops.Dropout(0.5, 1, row0=(1 << 32) - 3)), dip.E_RANGE)])
def test_linear_refusals(lib, change, code):
    a = linear(**change)
    assert lib.dip_linear(ctypes.byref(a), None) == code
    assert lib.dip_linear_workspace(ctypes.byref(a)) == code


def test_empty_calls_are_done(lib):
    for change in (dict(m=0, x=None, y=None), dict(n=0, w=None, y=None)):
        assert lib.dip_linear(ctypes.byref(linear(**change)), None) == dip.OK
    assert lib.dip_dropout_add(ops.F32, 0, 5, None, 0, None, 0, ctypes.byref(ops.Dropout(0.5, 1)), None, 0, None) == dip.OK
    assert lib.dip_linear(None, None) == dip.E_INVAL and lib.dip_linear_grad(None, None) == dip.E_INVAL
    assert lib.dip_group_norm(None, None) == dip.E_INVAL and lib.dip_group_norm_grad(None, None) == dip.E_INVAL


def grad(**kw):
    a = ops._LinearGrad(m=4, n=8, k=16, dtype=ops.BF16, dy=AT, ldy=8, x=AT, ldx=16, w=AT, ldw=16,
                        dx=AT, lddx=16, dw=AT, lddw=16, db=AT, grad_dtype=ops.BF16, workspace=AT,
                        workspace_bytes=1 << 20)
    for k, v in kw.items():
        setattr(a, k, v)
    return a


@pytest.mark.parametrize("change,code", [
    (dict(grad_dtype=ops.F16), dip.E_INVAL), (dict(act=ops.ACTS["silu"]), dip.E_INVAL), (dict(dy=None), dip.E_INVAL),
    (dict(x=None), dip.E_INVAL), (dict(w=None), dip.E_INVAL), (dict(lddx=15), dip.E_INVAL), (dict(lddw=8), dip.E_INVAL),
    (dict(grad_dtype=ops.F32, dw=AT + 2), dip.E_INVAL), (dict(grad_dtype=ops.F32, db=AT + 2), dip.E_INVAL),
    (dict(workspace_bytes=16), dip.E_CAPACITY), (dict(workspace=AT + 8), dip.E_INVAL), (dict(workspace=None), dip.E_INVAL),
    (dict(n=-1), dip.E_INVAL)])
def test_linear_grad_refusals(lib, change, code):
    assert lib.dip_linear_grad(ctypes.byref(grad(**change)), None) == code


@pytest.mark.parametrize("change,code", [
    (dict(groups=0), dip.E_INVAL), (dict(groups=5), dip.E_INVAL), (dict(eps=-1.0), dip.E_INVAL),
    (dict(eps=float("nan")), dip.E_INVAL), (dict(x=None), dip.E_INVAL), (dict(x_ss=11), dip.E_INVAL),
    (dict(x_sb=40), dip.E_INVAL), (dict(y_ss=0), dip.E_INVAL), (dict(gamma=AT + 1), dip.E_INVAL), (dict(mean=AT + 2), dip.E_INVAL),
    (dict(dtype=7), dip.E_INVAL), (dict(act=9), dip.E_INVAL), (dict(b=1 << 31), dip.E_RANGE)])
def test_group_norm_refusals(lib, change, code):
    a = ops._GroupNorm(b=2, s=4, c=12, groups=3, dtype=ops.F16, eps=1e-5, x=AT, x_sb=48, x_ss=12, y=AT, y_sb=48, y_ss=12)
    for k, v in change.items():
        setattr(a, k, v)
    assert lib.dip_group_norm(ctypes.byref(a), None) == code
    assert lib.dip_group_norm_workspace(ctypes.byref(a)) == code


@pytest.mark.parametrize("change,code", [
    (dict(mean=None), dip.E_INVAL), (dict(dy=None), dip.E_INVAL), (dict(dx_ss=3), dip.E_INVAL),
    (dict(dgamma=AT + 1), dip.E_INVAL), (dict(workspace_bytes=0), dip.E_CAPACITY), (dict(workspace=AT + 4), dip.E_INVAL)])
def test_group_norm_grad_refusals(lib, change, code):
    a = ops._GroupNormGrad(b=2, s=4, c=12, groups=3, dtype=ops.F16, dy=AT, dy_sb=48, dy_ss=12, x=AT, x_sb=48, x_ss=12,
                           mean=AT, rstd=AT, dx=AT, dx_sb=48, dx_ss=12, dgamma=AT, dbeta=AT, workspace=AT,
                           workspace_bytes=1 << 30)
    for k, v in change.items():
        setattr(a, k, v)
    assert lib.dip_group_norm_grad(ctypes.byref(a), None) == code

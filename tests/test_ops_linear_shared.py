"""Which products of a linear's gradients share a launch, by the workspace that a call
asks for: in one launch both products' partial sums lie beside each other, one after the
other they take the same place.  The sizes split the contraction of both products."""
import ctypes

import pytest

pytest.importorskip("torch")

from paper_2504_14145_amd import load
from paper_2504_14145_amd.ops import BF16, _LinearGrad


def workspace(m, k, n, dx=True, dw=True):
    lib = load()
    lib.dip_linear_grad_workspace.argtypes = [ctypes.c_void_p]
    lib.dip_linear_grad_workspace.restype = ctypes.c_int64
    a = _LinearGrad(m=m, n=n, k=k, dtype=BF16, grad_dtype=BF16, dy=1 << 20, ldy=n, x=2 << 20, ldx=k, w=3 << 20, ldw=k,
                    dx=4 << 20 if dx else None, lddx=k, dw=5 << 20 if dw else None, lddw=k)
    return lib.dip_linear_grad_workspace(ctypes.addressof(a))


def shared(m, k, n):
    x, w, both = workspace(m, k, n, dw=False), workspace(m, k, n, dx=False), workspace(m, k, n)
    assert x > 0 and w > 0 and both in (max(x, w), x + w)
    return both == x + w


@pytest.mark.parametrize("m,k,n", [(18176, 512, 7936), (12032, 768, 6912), (17664, 512, 7424), (11520, 768, 6912)])
def test_what_one_launch_slows_down_has_two(m, k, n):
    """Measured 11 to 23 % slower in one launch: 128 x 128 tiles in several rounds in the
    place of larger ones."""
    assert not shared(m, k, n)


@pytest.mark.parametrize("m,k,n", [(2880, 256, 1664), (3200, 576, 2688)])
def test_what_leaves_the_card_idle_shares_one(m, k, n):
    """Measured 18 to 27 % faster."""
    assert shared(m, k, n)

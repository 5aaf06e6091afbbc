"""Layouts that callers of the C ABI are compiled against."""
import ctypes

from paper_2504_14145_amd import ops


def test_offsets_stay():
    """A member that is added takes the place of padding: the others keep theirs."""
    at = {n: getattr(ops._GroupNormGrad, n).offset for n, _ in ops._GroupNormGrad._fields_}
    assert at["act"] == 32 and at["dy"] == 40 and at["dgamma"] == 144 and at["workspace"] == 160
    assert ctypes.sizeof(ops._GroupNormGrad) == 176
    assert ctypes.sizeof(ops._Linear) == 160 and ctypes.sizeof(ops._LinearGrad) == 184
    assert ctypes.sizeof(ops._GroupNorm) == 136

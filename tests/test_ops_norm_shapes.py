"""Group norm at shapes where a kernel's lanes or a sample's positions run out:
no positions, and (on the GPU) vectors that end inside a group."""
import ctypes
import subprocess
import sys

import pytest

torch = pytest.importorskip("torch")

from paper_2504_14145_amd import ops  # noqa: E402

CALL = """
import ctypes
from paper_2504_14145_amd import ops
lib = ops._load()
for c, groups in ((8, 1), (4096, 1), (4104, 1), (8192, 1), (8192, 2), (40000, 4)):
    a = ops._GroupNorm(b=3, s=0, c=c, groups=groups, dtype=ops.BF16)
    print(lib.dip_group_norm_workspace(ctypes.byref(a)) >= 0)
"""


def test_workspace_without_positions():
    """In a process of its own: a division by zero would end it."""
    out = subprocess.run([sys.executable, "-c", CALL], capture_output=True, text=True,
                         cwd=str(__import__("pathlib").Path(__file__).parent.parent))
    assert out.returncode == 0, out.stderr
    assert out.stdout.split() == ["True"] * 6


@pytest.mark.gpu
@pytest.mark.parametrize("c,groups", [(8, 1), (4104, 1), (40000, 4)])
def test_no_positions(c, groups):
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    x = torch.empty((3, 0, c), dtype=torch.bfloat16, device="cuda")
    y, mean, rstd = ops.group_norm(x, groups, eps=0.25)
    assert y.shape == x.shape and bool((mean == 0).all()) and bool((rstd == 2).all())

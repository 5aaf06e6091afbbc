"""Statements of the kernels' sources that the compiler does not check."""
import glob
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(__file__)), "paper_2504_14145_amd", "csrc")


def statements():
    for path in sorted(glob.glob(os.path.join(CSRC, "*.h*"))):
        for s in re.findall(r"asm volatile\((.*?)\);", open(path).read(), flags=re.S):
            yield os.path.basename(path), s


def test_m0_goes_from_statement_to_statement_as_a_value():
    """Between two statements the compiler may put M0 to its own uses: a load to LDS
    says that it takes M0, and M0 is written only as a statement's result."""
    loads = [(f, s) for f, s in statements() if re.search(r"buffer_load\w* .*\blds\b", s)]
    assert loads and all('"{m0}"(' in s for f, s in loads), loads
    for f, s in statements():
        text = "".join(re.findall(r'"((?:[^"\\]|\\.)*)"', s.split(":")[0]))
        assert not re.search(r"\bm0\b", text), (f, s)
    assert any('"={m0}"(' in s for f, s in statements())

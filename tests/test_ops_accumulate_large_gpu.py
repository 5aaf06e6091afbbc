"""Weight gradients of whole large tiles that are float32 or added to: the sizes at
which a layer block sums them."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from ops_reference import EPS32, assert_close  # noqa: E402

if torch.cuda.is_available():
    from paper_2504_14145_amd import ops

F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16


@pytest.fixture(autouse=True)
def need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


# 14 x 16 tiles of 256 x 256, one round of the card: whole ones, and ragged edges at
# odd strides
@pytest.mark.parametrize("m,n,k,pad", [(600, 3584, 4096, 0), (601, 3501, 3999, 0), (640, 3584, 4000, 3)])
@pytest.mark.parametrize("dtype,out,accumulate", [(BF16, F32, True), (BF16, F32, False), (BF16, BF16, True),
                                                  (F16, F32, True)])
def test_large_tiles_added_to(m, n, k, pad, dtype, out, accumulate):
    g = torch.Generator(device="cuda").manual_seed(n)
    x, dy = (torch.randn(s, generator=g, device="cuda").to(dtype) for s in ((m, k), (m, n)))
    w = torch.empty((n, k), dtype=dtype, device="cuda")
    old = torch.randn((n, k + pad), generator=g, device="cuda").to(out)
    dw = old.clone()
    _, got, _ = ops.linear_backward(dy, x, w, need_dx=False, bias=False, dw=dw[:, :k], accumulate=accumulate)
    assert got.data_ptr() == dw.data_ptr()
    t = dy.double().t().contiguous()
    want, size = t @ x.double(), t.abs() @ x.double().abs()
    start = old[:, :k].double() if accumulate else torch.zeros_like(want)
    bound = 2 * (m + 8) * EPS32 * size + 4 * EPS32 * (want.abs() + start.abs())
    assert_close(dw[:, :k], (want + start).cpu(), bound.cpu(), out, f"{dtype} {out}")
    assert torch.equal(dw[:, k:], old[:, k:]), "columns beyond k were written"

"""Tensors that require gradients: the operators record none and say so."""
import warnings

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

if torch.cuda.is_available():
    from paper_2504_14145_amd import ops


@pytest.fixture(autouse=True)
def need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


def test_a_forward_that_cuts_a_graph_warns():
    x, w, r = (torch.randn(s, device="cuda").bfloat16() for s in ((8, 16), (24, 16), (8, 24)))
    b, v, gamma = (torch.randn(s, device="cuda").bfloat16() for s in ((24,), (2, 5, 16), (16,)))
    drop = ops.Dropout(0.1, 1)

    def calls():
        return (("linear", lambda: ops.linear(x, w, b, residual=r), (x, w, b, r)),
                ("dropout_add", lambda: ops.dropout_add(x, drop, x), (x,)),
                ("group_norm", lambda: ops.group_norm(v, 4, gamma, gamma)[0], (v, gamma)))

    for name, call, given in calls():
        want = call()
        for t in given:
            t.requires_grad_(True)
            with pytest.warns(UserWarning, match=f"{name} records no gradients"):
                got = call()
            assert torch.equal(got, want) and not got.requires_grad
            with warnings.catch_warnings():
                warnings.simplefilter("error")
                with torch.no_grad():
                    assert torch.equal(call(), want)
                if name == "linear":    # the caller's own backward
                    ops.linear_backward(r.detach(), x, w)
            t.requires_grad_(False)
        with warnings.catch_warnings():
            warnings.simplefilter("error")
            call()

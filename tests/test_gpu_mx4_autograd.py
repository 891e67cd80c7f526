"""Dropout and a product of microscaled 4-bit floats as autograd functions around the library's calls, and what is refused outside of them."""
import pytest
import torch

from tests.test_gpu_mx4 import b, draw, matrix  # noqa: F401  (b: a fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_refused_where_gradients_are_recorded(b, dtype):
    x, r = matrix(8, 64, dtype), matrix(8, 64, dtype, 1)
    leaf, rleaf = x.clone().requires_grad_(), r.clone().requires_grad_()
    for call in (lambda: b.dropout(leaf, 0.5, draw(b)), lambda: b.dropout(leaf * 1, 0.5, draw(b)), lambda: b.dropout(x, 0.5, draw(b), add=rleaf),
                 lambda: b.dropout(leaf, 0.5, draw(b), add=r), lambda: b.dropout(x, 0.5, draw(b), out=rleaf), lambda: b.mx4_quantise(leaf)):
        with pytest.raises(b.ConEFError, match="gradient"):
            call()
    want = b.dropout(x, 0.5, draw(b), add=r), b.mx4_quantise(x)
    with torch.no_grad():
        got = b.dropout(leaf, 0.5, draw(b), add=rleaf), b.mx4_quantise(leaf)
        assert torch.equal(b.dropout(leaf, 0.5, draw(b)), b.dropout(x, 0.5, draw(b)))
    assert torch.equal(got[0], want[0]) and torch.equal(got[1].codes, want[1].codes) and torch.equal(got[1].scales, want[1].scales)
    assert torch.equal(b.dropout(leaf.detach(), 0.5, draw(b)), b.dropout(x, 0.5, draw(b)))


def test_in_an_autograd_function(b):
    """y = dropout(x) + r: gradients are the same call and the gradient itself."""
    class Drop(torch.autograd.Function):
        @staticmethod
        def forward(ctx, x, r):
            return b.dropout(x, 0.25, draw(b), add=r)

        @staticmethod
        def backward(ctx, dy):
            return b.dropout(dy, 0.25, draw(b)), dy

    x, r = (matrix(20, 77, torch.float32, s).requires_grad_() for s in range(2))
    dy = matrix(20, 77, torch.float32, 2)
    Drop.apply(x, r).backward(dy)
    assert torch.equal(x.grad, b.dropout(dy, 0.25, draw(b))) and torch.equal(r.grad, dy)

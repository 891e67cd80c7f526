"""Gradients of a norm's weight over so many rows that sums of 32 bits along all rows of a thread block would show."""
import pytest
import torch

from tests.test_gpu_f8 import b, matrix  # noqa: F401  (b: a fixture)

pytestmark = pytest.mark.gpu


def bound(rows, count):
    """Of sums of `count` equal terms a row: 256 rows and a block's eight warps in 32 bits, half a step of 2^-23 each; the rest in 64, rounded once."""
    return (min(rows, 256) + 8 + 1) * 2.0 ** -24 * rows * count


@pytest.mark.parametrize("rows,cols", [(20_000_003, 4), (20_000_003, 3), (20_000_003, 1)])
def test_equal_terms(b, rows, cols):
    """A term whose sum in 32 bits falls behind by the same part of a step each time: 4223 rows to a warp are off by 6e-5 in one chain."""
    term = 1.0159916877746582
    dy, h = torch.full((rows, cols), term, device="cuda"), torch.ones(rows, cols, device="cuda")
    _, dw = b.rms_norm_grad(dy, h, torch.ones(cols, device="cuda"), torch.ones(rows, device="cuda"))
    assert ((dw.double() - term * rows).abs() <= bound(rows, term)).all(), dw / (term * rows) - 1


@pytest.mark.parametrize("rows,cols,dtype", [(1_300_000, 100, torch.bfloat16), (650_001, 257, torch.bfloat16), (650_001, 264, torch.float16), (1_300_001, 8, torch.float32)])
def test_every_row_counts_once(b, rows, cols, dtype):
    """Against the products in 64 bits; and each row alone, without the others."""
    dy, h = matrix(rows, cols, dtype), matrix(rows, cols, dtype, 1)
    w, rstd = torch.ones(cols, device="cuda"), torch.rand(rows, device="cuda") + 0.5
    _, dw = b.rms_norm_grad(dy, h, w, rstd)
    want, size = torch.zeros(2, cols, dtype=torch.float64, device="cuda")
    for r in range(0, rows, 100_000):
        p = dy[r:r + 100_000].double() * h[r:r + 100_000].double() * rstd[r:r + 100_000, None].double()
        want += p.sum(0)
        size += p.abs().sum(0)
    # a term's two roundings, its chain's 256 (and eight), the last one's
    assert ((dw.double() - want).abs() <= size * (2 + 256 + 8) * 2.0 ** -24 + want.abs() * 2.0 ** -24).all()
    again = b.rms_norm_grad(dy, h, w, rstd)[1]
    assert torch.equal(again, dw)
    one = torch.zeros_like(dy)
    for row in (0, 255, 256, rows // 3, rows - 1):
        one[row] = dy[row]
        n = h[row].float() * rstd[row]
        assert torch.equal(b.rms_norm_grad(one, h, w, rstd)[1], dy[row].float() * n)
        one[row] = 0


def test_long_rows(b):
    """... of more columns than a group, 473 rows to a block, more than 2^31 elements."""
    rows, cols = 70000, 32768
    gen = torch.Generator(device="cuda")
    gen.manual_seed(8)
    block = torch.randn(1000, cols, generator=gen, device="cuda").bfloat16()
    h = block.repeat(rows // 1000, 1)
    dy = h.flip(1)
    rstd = torch.rand(rows, generator=gen, device="cuda") + 0.5
    dw = b.rms_norm_grad(dy, h, torch.ones(cols, device="cuda"), rstd)[1]
    p = block.double() * block.flip(1).double()
    each = rstd.view(-1, 1000).double().sum(0)[:, None]
    want, size = (p * each).sum(0), (p * each).abs().sum(0)
    assert ((dw.double() - want).abs() <= size * (2 + 256 + 8) * 2.0 ** -24 + want.abs() * 2.0 ** -24).all()

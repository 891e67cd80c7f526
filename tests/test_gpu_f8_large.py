"""8-bit forms, norms and products of more than 2^31 elements: the last rows are those of a small matrix."""
import pytest
import torch

from tests.test_gpu_f8 import b  # noqa: F401  (a fixture)

pytestmark = pytest.mark.gpu

ROWS, COLS, LAST = 70000, 32768, 300


@pytest.fixture(scope="module")
def x():
    gen = torch.Generator(device="cuda")
    gen.manual_seed(5)
    block = torch.randn(1000, COLS, generator=gen, device="cuda").bfloat16()
    big = block.repeat(ROWS // 1000, 1)
    big += (torch.arange(ROWS, device="cuda") % 7).bfloat16()[:, None]
    yield big
    del big
    torch.cuda.empty_cache()


def rows_of(form, first, rows):
    """The codes of some rows."""
    pitch = (form.cols + 127) // 128 * 128
    return form.codes.view(form.rows, pitch)[first:first + rows]


def test_forms_and_values(b, x):
    tail = x[-LAST:].contiguous()
    r, t = b.f8_quantise(x, "both")
    small = b.f8_quantise(tail)
    assert torch.equal(rows_of(r, ROWS - LAST, LAST), rows_of(small, 0, LAST))
    assert torch.equal(b.f8_dequantise(r, torch.bfloat16)[-LAST:], b.f8_dequantise(small, torch.bfloat16))
    column = b.f8_quantise(x[:, -3:].contiguous(), "cols")
    assert torch.equal(rows_of(t, COLS - 3, 3), rows_of(column, 0, 3))
    alone = b.f8_quantise(x)
    assert torch.equal(alone.codes, r.codes) and torch.equal(alone.scales, r.scales)


def test_norm_and_gradient(b, x):
    w = torch.ones(COLS, device="cuda") * 1.5
    tail = x[-LAST:].contiguous()
    out, small = b.rms_norm(x, w, 1e-5, add=x), b.rms_norm(tail, w, 1e-5, add=tail)
    assert torch.equal(out.y[-LAST:], small.y) and torch.equal(out.h[-LAST:], small.h) and torch.equal(out.rstd[-LAST:], small.rstd)
    dx, _ = b.rms_norm_grad(out.y, out.h, w, out.rstd, add=x)
    few, _ = b.rms_norm_grad(small.y, small.h, w, small.rstd, add=tail)
    assert torch.equal(dx[-LAST:], few)
    del dx, few
    forms = b.rms_norm(x, w, 1e-5, forms="rows").y
    assert torch.equal(rows_of(forms, ROWS - LAST, LAST), rows_of(b.rms_norm(tail, w, 1e-5, forms="rows").y, 0, LAST))


def test_rows_of_a_wider_matrix(b, x):
    """Rows 2^31 elements and more from the first, that are not one array."""
    view, tail = x[:, 8:1008], x[-LAST:, 8:1008]
    w = torch.ones(1000, device="cuda")
    assert torch.equal(b.rms_norm(view, w).y[-LAST:], b.rms_norm(tail.contiguous(), w).y)
    assert torch.equal(rows_of(b.f8_quantise(view), ROWS - LAST, LAST), rows_of(b.f8_quantise(tail.contiguous()), 0, LAST))
    odd = x[:, 7:1006]
    assert torch.equal(b.rms_norm(odd, w[:999]).y[-LAST:], b.rms_norm(odd[-LAST:].contiguous(), w[:999]).y)


def test_product(b, x):
    a, c = x[:, :96].contiguous(), x[:COLS, 96:192].contiguous()
    fa, fc = b.f8_quantise(a), b.f8_quantise(c)
    out = b.f8_matmul(fa, fc)
    assert torch.equal(out[-LAST:], b.f8_matmul(b.f8_quantise(a[-LAST:].contiguous()), fc))


def test_gradient_of_a_row_with_more_than_2_29_columns(b):
    """More groups of columns than a grid's second dimension has blocks.  The row repeats a pattern, so the formula's mean is the pattern's."""
    period, repeats = 1 << 16, 8194   # 65552 groups of 8192 columns
    gen = torch.Generator(device="cuda")
    gen.manual_seed(6)
    dy, h, w = ((torch.randn(period, generator=gen, device="cuda") + 0.5).bfloat16() for _ in range(3))
    rstd = torch.full((1,), 0.75, device="cuda")
    dx, dw = b.rms_norm_grad(dy.repeat(repeats)[None], h.repeat(repeats)[None], w.repeat(repeats), rstd)
    n, g = h.double() * 0.75, dy.double() * w.double()
    mean, size = (g * n).mean(), (g * n).abs().mean()
    want = 0.75 * (g - n * mean)
    # the mean: 8 terms of three roundings each in 32 bits, the rest in 64; two more to multiply it, three of the difference, and dx's own to 8 bits
    loose = 0.75 * (n.abs() * size * 14 + (g.abs() + n.abs() * mean.abs()) * 4) * 2.0**-24
    for part in (dx[0, :period], dx[0, period * 4097:period * 4098], dx[0, -period:]):
        assert ((part.double() - want).abs() <= want.abs() * 2.0**-8 + loose * (1 + 2.0**-8)).all()
    for part in (dw[:period], dw[-period:]):
        assert ((part.double() - dy.double() * n).abs() <= (dy.double() * n).abs() * 2.0**-23).all()

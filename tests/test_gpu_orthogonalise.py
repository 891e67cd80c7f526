"""Orthogonalised updates against the same products in 64 bits."""
import numpy as np
import pytest
import torch

from oracle import f8_oracle as fo
from tests.test_gpu_f8 import DTYPES, EPS, b, f64, matrix  # noqa: F401  (b: a fixture)

pytestmark = pytest.mark.gpu

QUINTIC = (3.4445, -4.7750, 2.0315)
CUBIC = (1.5, -0.5, 0.0)


def update(rows, cols, dtype, seed=0, rank=None, noise=0.1):
    """A part of low rank and noise in all directions, small as gradients are."""
    gen = torch.Generator(device="cuda")
    gen.manual_seed(rows * 10007 + cols + seed)
    rank = rank or max(1, min(rows, cols) // 8)
    x = torch.randn(rows, rank, generator=gen, device="cuda") @ torch.randn(rank, cols, generator=gen, device="cuda") / rank ** 0.5
    return ((x + noise * torch.randn(rows, cols, generator=gen, device="cuda")) * 1e-3).to(dtype)


def check(got, x, steps=5, coefficients=QUINTIC, scale=1.0):
    """Rounding to the type is off by half a step at most.  Operands are kept to 2^-23 of their size (the half of fp16's lower part) and
    sums in fp32: each step's X is off by 2^-20 relative at most, and the steps behind raise that by their slope at zero each, which is the largest.  (From 256 rows on
    some products take 11 bits, which adds 1.2e-3 at most; in the norm rounding loses 2^-8 / sqrt(3) / 1.4 = 1.7e-3, their root of squares is 2.0e-3, and 2^-8 is 3.9e-3.  For
    float16, from 512 rows on, 2.7e-4 and 2.1e-4 are 3.4e-4 of 4.9e-4.)"""
    want = fo.orthogonalise(f64(x), steps, coefficients, scale)
    tol = EPS[got.dtype] + 2.0 ** -20 * sum(abs(coefficients[0]) ** i for i in range(1, steps + 1))
    far = np.linalg.norm(f64(got) - want) / max(np.linalg.norm(want), 1e-300)
    assert got.shape == x.shape and far <= tol, (far, tol)


SHAPES = [(1, 1), (1, 7), (7, 1), (2, 2), (5, 64), (64, 5), (33, 130), (128, 128), (129, 127), (127, 400), (256, 512), (513, 250), (300, 1301)]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows,cols", SHAPES)
def test_matrices(b, rows, cols, dtype):
    x = update(rows, cols, dtype)
    for to in (torch.bfloat16, torch.float16):
        check(b.orthogonalise(x, dtype=to), x)
    check(b.orthogonalise(x, steps=1, scale=-0.25), x, 1, scale=-0.25)
    check(b.orthogonalise(x, steps=8, coefficients=CUBIC, dtype=torch.float16), x, 8, CUBIC)


@pytest.mark.parametrize("rows,cols,batch", [(1600, 1600, 1), (700, 2500, 3), (2500, 700, 2), (1100, 1100, 5), (40, 50, 30), (256, 256, 40)])
def test_large_and_many(b, rows, cols, batch):
    x = torch.stack([update(rows, cols, torch.bfloat16, i) for i in range(batch)])
    got = b.orthogonalise(x)
    for i in range(0, batch, max(1, batch // 3)):
        check(got[i], x[i])
    assert torch.equal(b.orthogonalise(x), got)
    if rows * cols < 10 ** 6:   # one alone: the same bits where its tiles are alike
        check(b.orthogonalise(x[batch - 1]), x[batch - 1])


@pytest.mark.parametrize("rows,cols,batch", [(1, 9000, 1), (100, 4000, 1), (40, 9001, 2), (300, 5000, 1), (128, 8192, 3), (5000, 130, 1), (3000, 200, 14), (513, 2500, 1)])
def test_long_rows(b, rows, cols, batch):
    """... whose products with themselves blocks share along the rows."""
    x = torch.stack([update(rows, cols, torch.bfloat16, i) for i in range(batch)])
    for to in (torch.bfloat16, torch.float16):
        got = b.orthogonalise(x, dtype=to)
        for i in {0, batch - 1}:
            check(got[i], x[i])
        assert all(torch.equal(b.orthogonalise(x, dtype=to), got) for _ in range(3))


def test_singular_values(b):
    """Those of the result are the polynomial of x's: no further from it than the result is from the exact one (Weyl), by check()'s bound.  (After twelve cubic
    steps the smallest of x, times 1.5 each, are still on their way to one.)"""
    x = matrix(200, 600, torch.float32)
    first = torch.linalg.svdvals(x.double()) / x.double().norm()
    for steps, (a, c3, c5), dtype in ((5, QUINTIC, torch.bfloat16), (12, CUBIC, torch.float16)):
        s = first
        for _ in range(steps):
            s = a * s + c3 * s ** 3 + c5 * s ** 5
        got = torch.linalg.svdvals(b.orthogonalise(x, steps=steps, coefficients=(a, c3, c5), dtype=dtype).double())
        tol = (EPS[dtype] + 2.0 ** -20 * sum(a ** i for i in range(1, steps + 1))) * s.norm()
        assert (got - s.sort(descending=True).values).abs().max() <= tol


@pytest.mark.parametrize("dtype", DTYPES)
def test_zeros_infinities_and_nan(b, dtype):
    x = torch.stack([update(70, 150, dtype, i) for i in range(5)])
    good = b.orthogonalise(x)
    x[1] = 0
    x[2, 3, 4] = float("inf")
    x[3, 69, 149] = float("nan")
    got = b.orthogonalise(x)
    assert not got[1].any() and torch.isnan(got[2]).all() and torch.isnan(got[3]).all()
    assert torch.equal(got[0], good[0]) and torch.equal(got[4], good[4])


def test_any_size_of_values(b):
    x = update(60, 90, torch.float32)
    want = b.orthogonalise(x)
    for scale in (2.0 ** 100, 2.0 ** -100):
        assert torch.equal(b.orthogonalise(x * scale), want)
    one = torch.zeros(40, 50, device="cuda")
    one[7, 9] = 1e30
    check(b.orthogonalise(one), one)


@pytest.mark.parametrize("rows,cols", [(60, 90), (90, 60)])
def test_strides_and_leading_dimensions(b, rows, cols):
    wide = torch.full((2, 3, rows + 5, cols + 9), 7.0, dtype=torch.bfloat16, device="cuda")
    x = wide[:, :, 2:2 + rows, 3:3 + cols]
    for i in range(2):
        for j in range(3):
            x[i, j] = update(rows, cols, torch.bfloat16, 3 * i + j)
    want = b.orthogonalise(x.contiguous())
    assert torch.equal(b.orthogonalise(x), want)
    out = torch.full_like(wide, 5.0)
    view = out[:, :, 1:1 + rows, 4:4 + cols]
    assert b.orthogonalise(x, out=view) is view
    assert torch.equal(view, want)
    view.fill_(5.0)
    assert (out == 5).all()
    y = x.contiguous()
    b.orthogonalise(y, out=y)
    assert torch.equal(y, want)
    b.orthogonalise(x, out=x)
    assert torch.equal(x, want)
    x.fill_(7.0)
    assert (wide == 7).all()
    assert torch.equal(b.orthogonalise(want[0, :, None]), b.orthogonalise(want[0].contiguous()).unsqueeze(1))


def test_nothing_in_it(b):
    for shape in ((0, 4), (4, 0), (0, 3, 4), (2, 0, 3)):
        assert b.orthogonalise(torch.empty(shape, device="cuda")).shape == shape


def test_streams_and_graphs(b):
    x = torch.stack([update(300, 200, torch.float32, i) for i in range(2)])
    want = b.orthogonalise(x)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    other = b.orthogonalise(x, stream=s)
    s.synchronize()
    assert torch.equal(other, want)
    torch.cuda.synchronize()
    graphs = []
    for i in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            out = b.orthogonalise(x[i])
        graphs.append((g, out))
    for seed in range(2):
        x.copy_(torch.stack([update(300, 200, torch.float32, 5 + seed + i) for i in range(2)]))
        for g, _ in graphs:
            g.replay()
        assert torch.equal(torch.stack([o for _, o in graphs]), torch.stack([b.orthogonalise(v) for v in x]))


def test_refusals(b):
    x = update(40, 60, torch.float32)
    bad = [lambda: b.orthogonalise(x[0]), lambda: b.orthogonalise(x, dtype=torch.float32), lambda: b.orthogonalise(x, out=torch.empty_like(x)), lambda: b.orthogonalise(x, steps=0),
           lambda: b.orthogonalise(x, steps=40), lambda: b.orthogonalise(x, coefficients=(1.0, 2.0)), lambda: b.orthogonalise(x, coefficients=(9.0, 9.0, 9.0)),
           lambda: b.orthogonalise(x.t()), lambda: b.orthogonalise(x.clone().requires_grad_()), lambda: b.orthogonalise(x, scale=float("nan")), lambda: b.orthogonalise(x.long()),
           lambda: b.orthogonalise(torch.zeros(5, 4, 6, 8, device="cuda")[:, 1:3]), lambda: b.orthogonalise(x.expand(3, 40, 60))]
    for call in bad:
        with pytest.raises(b.ConEFError) as e:
            call()
        assert e.value.code == b.ERR_INVALID_ARG


def test_nothing_runs_out(b):
    before = b.orthogonalise_timeouts()
    assert not torch.isnan(b.orthogonalise(update(700, 1300, torch.bfloat16))).any()
    assert b.orthogonalise_timeouts() == before

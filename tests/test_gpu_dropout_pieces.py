"""Dropout and rows to microscaled 4-bit floats at sizes where a thread takes several pieces, and the sign of zeros wherever they lie."""
import numpy as np
import pytest
import torch

from oracle import mx4_oracle as mo
from tests.test_gpu_mx4 import DTYPES, SEED, b, check_dropout, draw, matrix, reference, strided, unpacked  # noqa: F401  (b: a fixture)

pytestmark = pytest.mark.gpu


def moved(t, by):
    """The same matrix as one array that begins `by` elements behind a boundary."""
    whole = torch.full((t.numel() + by + 9,), 7.0, dtype=t.dtype, device="cuda")
    whole[by:by + t.numel()] = t.reshape(-1)
    return whole[by:by + t.numel()].view(t.shape), whole


# ------------------------------------------------------------------ zeros

@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows,cols", [(8, 64), (1, 1003), (40, 33), (3, 1301), (50, 2), (7, 1), (9, 2500)])
def test_a_kept_zero_has_its_own_sign_wherever_it_lies(b, rows, cols, dtype):
    """Kept elements are multiplied, so -0 stays -0; dropped ones are +0.  With a residual the sum decides: -0 where both are, else +0."""
    zeros = torch.where(torch.arange(rows * cols, device="cuda").view(rows, cols) % 3 == 0, 0.0, -0.0).to(dtype)
    kept = torch.from_numpy(mo.numbers(*SEED, rows, cols, mo.DROPOUT) >= 32768).cuda()
    r = torch.where(torch.arange(rows * cols, device="cuda").view(rows, cols) % 5 < 2, 0.0, -0.0).to(dtype)
    neg, rneg = torch.signbit(zeros), torch.signbit(r)
    out = strided(zeros, 0, 5)[0]
    for x in (zeros, moved(zeros, 1)[0], moved(zeros, 3)[0], strided(zeros, 0, 8)[0], strided(zeros, 1, 3)[0], strided(zeros, 5, 2)[0]):
        for y in (b.dropout(x, 0.5, draw(b)), b.dropout(x, 0.5, draw(b), out=out)):
            assert not y.any() and torch.equal(torch.signbit(y), kept & neg)
        y = b.dropout(x, 0.5, draw(b), add=r)
        assert not y.any() and torch.equal(torch.signbit(y), torch.where(kept, neg & rneg, rneg))


# ------------------------------------------------------------------ several pieces per thread

@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("by", [0, 1, 6])
@pytest.mark.parametrize("rows,cols", [(5000, 1301), (2500001, 2)])
def test_dropout_of_large_arrays_of_any_width(b, rows, cols, dtype, by):
    x = moved(matrix(rows, cols, dtype), by)[0]
    check_dropout(b.dropout(x, 0.35, draw(b), out=moved(x, by)[0]), x, 0.35)
    r, (y, whole) = moved(matrix(rows, cols, dtype, 1), by)[0], moved(x, by)
    check_dropout(b.dropout(x, 0.35, draw(b), add=r, out=y), x, 0.35, r)
    assert (whole[:by] == 7).all() and (whole[by + rows * cols:] == 7).all()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows,cols", [(4000, 1600), (1, 5000003)])
def test_dropout_of_large_arrays_of_whole_groups(b, rows, cols, dtype):
    x, r = matrix(rows, cols, dtype), matrix(rows, cols, dtype, 1)
    check_dropout(b.dropout(x, 0.1, draw(b)), x, 0.1)
    check_dropout(b.dropout(x, 0.1, draw(b), add=r), x, 0.1, r)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("front", [0, 3])
def test_dropout_of_rows_in_several_runs(b, dtype, front):
    """Rows longer than a warp walks at a time, of a wider matrix."""
    x = matrix(5, 30007, dtype)
    xs, (y, wide) = strided(x, front, 5)[0], strided(x, front, 5)
    check_dropout(b.dropout(xs, 0.3, draw(b), out=y), x, 0.3)
    assert (wide[:, :front] == 7).all() and (wide[:, front + 30007:] == 7).all()


def test_dropout_of_many_rows_that_begin_differently(b):
    """More groups of four columns than the threads of a launch that takes them one by one."""
    x = matrix(2500, 4001, torch.bfloat16)
    xs, (y, wide) = strided(x, 1, 2)[0], strided(x, 2, 5)
    check_dropout(b.dropout(xs, 0.3, draw(b), out=y), x, 0.3)
    assert (wide[:, :2] == 7).all() and (wide[:, -5:] == 7).all()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("stochastic,p", [(False, 0.0), (True, 0.0), (False, 0.3), (True, 0.3)])
def test_rows_of_many_blocks(b, dtype, stochastic, p):
    x = matrix(4000, 1600, dtype)
    x[5, 70], x[3999, 1599], x[17, :64] = float("inf"), float("nan"), -0.0
    codes, scales = unpacked(b.mx4_quantise(x, stochastic=stochastic, p=p, draw=draw(b)))
    want = reference(x, stochastic, p, False)
    assert np.array_equal(scales, want[1]) and np.array_equal(codes, want[0])

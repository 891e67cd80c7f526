"""Stacks of matrices that lie between one another's rows, as parts of a wider weight do."""
import pytest
import torch

from tests.test_gpu_f8 import DTYPES, b  # noqa: F401  (b: a fixture)
from tests.test_gpu_orthogonalise import update

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows,cols,parts,gap", [(60, 96, 2, 0), (96, 60, 3, 0), (130, 64, 3, 8), (33, 50, 4, 1), (1, 40, 2, 0), (300, 256, 3, 0)])
def test_parts_of_a_wider_matrix(b, rows, cols, parts, gap, dtype):
    wide = torch.full((rows, parts * (cols + gap)), 7.0, dtype=dtype, device="cuda")
    x = wide.view(rows, parts, cols + gap)[:, :, :cols].transpose(0, 1)
    for i in range(parts):
        x[i] = update(rows, cols, dtype, i)
    to = torch.float16 if dtype == torch.float16 else torch.bfloat16
    want = b.orthogonalise(x.contiguous())
    assert want.dtype == to and torch.equal(b.orthogonalise(x), want)
    out = torch.full((rows, parts * (cols + gap)), 5.0, dtype=to, device="cuda")
    view = out.view(rows, parts, cols + gap)[:, :, :cols].transpose(0, 1)
    assert b.orthogonalise(x, out=view) is view and torch.equal(view, want)
    view.fill_(5.0)
    assert (out == 5).all()
    if dtype == to:
        b.orthogonalise(x, out=x)
        assert torch.equal(x, want)
        x.fill_(7.0)
        assert (wide == 7).all()


def test_shared_elements_are_refused(b):
    big = torch.zeros(400, device="cuda")
    for size, strides in (((2, 4, 8), (7, 16, 1)), ((2, 4, 8), (9, 16, 1)), ((3, 4, 8), (8, 16, 1))):
        with pytest.raises(b.ConEFError) as e:
            b.orthogonalise(big.as_strided(size, strides))
        assert e.value.code == b.ERR_INVALID_ARG

"""Distances between the matrices of a stack to orthogonalise, as the library checks them (nothing is launched: the workspace is too small)."""
import ctypes as C

import pytest

P = 1 << 20


@pytest.fixture(scope="module")
def b():
    from paper_2312_08538_b200 import binding
    return binding


def code(b, batch, rows, cols, x=None, out=None):
    """... of stacks with (ld, stride)."""
    (ld, stride), (out_ld, out_stride) = x or (cols, rows * cols), out or (cols, rows * cols)
    return b.lib.conef_orthogonalise(P, b.BF16, batch, rows, cols, ld, stride, 5, (C.c_double * 3)(3.4445, -4.7750, 2.0315), 1.0, P, b.BF16, out_ld, out_stride, None, 0, None)


def test_matrices_that_share_nothing_are_taken(b):
    for at in ((8, 32), (8, 40), (20, 68), (16, 8), (17, 8), (18, 10), (1 << 20, 500000)):   # 2 x 4 x 8
        assert code(b, 2, 4, 8, x=at) == code(b, 2, 4, 8, out=at) == b.ERR_WORKSPACE_TOO_SMALL
    for at in ((24, 8), (32, 12)):
        assert code(b, 3, 4, 8, x=at) == code(b, 3, 4, 8, out=at) == b.ERR_WORKSPACE_TOO_SMALL
    assert code(b, 3, 1, 8, x=(8, 8)) == b.ERR_WORKSPACE_TOO_SMALL


def test_matrices_that_share_elements_are_refused(b):
    for at in ((8, 31), (8, 8), (16, 7), (15, 8), (16, 9), (16, 0), (16, -8), (20, 67)):
        assert code(b, 2, 4, 8, x=at) == code(b, 2, 4, 8, out=at) == b.ERR_INVALID_ARG
    for at in ((24, 9), (16, 8), (31, 12), (24, 7)):
        assert code(b, 3, 4, 8, x=at) == code(b, 3, 4, 8, out=at) == b.ERR_INVALID_ARG

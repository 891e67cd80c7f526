"""Values of 8-bit forms whose scales are next to the smallest, 2^-127: exact in float32, rounded to nearest even in bfloat16, whose last place is 2^-133, and in float16."""
import numpy as np
import pytest
import torch

from oracle import f8_oracle as fo
from tests.test_gpu_f8 import KINDS, b, f64  # noqa: F401  (b: a fixture)

pytestmark = pytest.mark.gpu
_LAST = {torch.bfloat16: -133, torch.float16: -24}


def nearest(v, last):
    """To multiples of 2^last, ties to even: what a type's subnormal numbers are."""
    return np.ldexp(np.round(np.ldexp(v, -last)), last)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("cols", [256, 261])
def test_values_of_the_smallest_scales(b, kind, cols):
    g = fo.grid(kind)
    rows = []
    for e in range(-127, -114):   # every code of the type under each scale, a block each
        block = np.zeros(cols)
        block[:g.size], block[128:128 + g.size] = g, -g
        rows.append(np.ldexp(block, e))
    x = np.array(rows)
    form = b.f8_quantise(torch.from_numpy(x).float().cuda(), kind=kind)   # (its elements are representable: exact)
    want = fo.decode(*fo.encode(x, kind), kind)
    assert np.array_equal(want, x) and np.array_equal(f64(b.f8_dequantise(form)), x)
    got = f64(b.f8_dequantise(form, torch.bfloat16))
    small = np.abs(x) < 2.0 ** -126
    assert np.array_equal(got[small], nearest(x[small], _LAST[torch.bfloat16])) and np.array_equal(got[~small], x[~small])
    assert np.array_equal(got[3 if kind == "e4m3" else 10:], x[3 if kind == "e4m3" else 10:]) and not np.array_equal(got[0], x[0])
    assert np.array_equal(f64(b.f8_dequantise(form, torch.float16)), nearest(x, _LAST[torch.float16]))

"""What the rounding of orthogonalised updates leaves to see of errors ahead of it, and that it tells operands of 22 bits from operands of 11 (here, in numpy, with
mistakes planted; the library's results: test_gpu_orthogonalise_precision.py)."""
import numpy as np
import pytest
import torch

from oracle import f8_oracle as fo

QUINTIC = (3.4445, -4.7750, 2.0315)
_BITS = {torch.bfloat16: 8, torch.float16: 11}   # of the significand


def beyond_rounding(got, want, dtype):
    """How far `got` lies from `want` (both float64) beyond half a step of the type, relative to want's size.  Where got is v rounded to nearest, each element is
    |v - want| beyond that at most, so this is no more than v's own error, however coarse the type is."""
    power = np.frexp(np.maximum(np.abs(got), np.abs(want)))[1] - 1
    half = np.ldexp(1.0, np.maximum(power, -126 if dtype == torch.bfloat16 else -14) - _BITS[dtype])
    return np.linalg.norm(np.maximum(np.abs(got - want) - half, 0.0)) / np.linalg.norm(want)


def tolerance(steps):
    """Of results before their rounding.  A product's operands are kept to 2^-23 each and the product of their lower parts, 2^-22, is left out; its sums, of three products
    each, lose a step of 2^-23 at most, a quarter of that on average over sums that grow, with every 16 elements along k: 3 k / 16 times 2^-25, for k = 2600 1.5e-5.  Three products a
    step, of which those of the last steps count (the ones before are raised, and with them the size of X): 4.4e-5 < 2^-14.  Steps around one neither raise nor lower
    errors much (slopes of -1.6 to 0.6): ten of them add up to less than twice that, of which half is beyond_rounding; behind twenty, whose slopes multiply, errors
    have been seen to grow eightfold in the same arithmetic: 2^-12."""
    return 2.0 ** -14 if steps <= 10 else 2.0 ** -12


def near_flat(rows, cols, seed):
    return np.random.default_rng(seed).standard_normal((rows, cols))


def decaying(rows, cols, seed):
    """Directions of sizes that fall off as 1 / i, as a momentum's do."""
    rng = np.random.default_rng(seed)
    n = min(rows, cols)
    u, v = (np.linalg.qr(rng.standard_normal((s, n)))[0] for s in (rows, cols))
    return u * (1.0 / np.arange(1, n + 1)) @ v.T


def orthogonalised(x, steps, bits):
    """The same products of operands rounded to so many bits, each under its own power of two; sums in 64 bits."""
    a, b, c = QUINTIC

    def cut(m):
        step = np.ldexp(1.0, np.frexp(m)[1] - bits)
        return np.round(m / step) * step

    y = x / np.linalg.norm(x)
    for _ in range(steps):
        g = cut(y) @ cut(y).T
        y = a * y + cut(b * g + c * (cut(g) @ cut(g))) @ cut(y)
    return y


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("steps", [5, 6, 10])
def test_bound_tells_22_bits_from_11(dtype, steps):
    for x in (near_flat(256, 320, steps), decaying(256, 320, steps)):
        want = fo.orthogonalise(x, steps, QUINTIC)
        for bits, passes in ((22, True), (11, False)):
            got = torch.from_numpy(orthogonalised(x, steps, bits)).float().to(dtype).double().numpy()
            assert (beyond_rounding(got, want, dtype) <= tolerance(steps)) == passes

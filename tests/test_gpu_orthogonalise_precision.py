"""Orthogonalised updates are as exact as their operands' 22 bits and sums of 32 make them, at any size and number of steps: what is beyond the result's own rounding."""
import numpy as np
import pytest
import torch

from oracle import f8_oracle as fo
from tests.test_gpu_f8 import b  # noqa: F401  (a fixture)
from tests.test_orthogonalise_precision import QUINTIC, beyond_rounding, decaying, near_flat, tolerance

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("rows,cols,steps", [(128, 300, 5), (256, 256, 5), (256, 512, 5), (256, 512, 6), (256, 512, 10), (256, 512, 20), (300, 1301, 6), (700, 512, 5), (512, 512, 20), (1024, 1100, 5),
                                             (513, 2600, 10)])
def test_results_before_their_rounding(b, rows, cols, steps, dtype):
    for make in (near_flat, decaying):
        x = torch.from_numpy(make(rows, cols, steps)).float()
        want = fo.orthogonalise(x.double().numpy(), steps, QUINTIC)
        got = b.orthogonalise(x.cuda(), steps=steps, dtype=dtype).double().cpu().numpy()
        far = beyond_rounding(got, want, dtype)
        assert far <= tolerance(steps), (far, tolerance(steps))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("rows,cols,steps", [(256, 16384, 5), (1024, 16384, 10), (6400, 1600, 5), (1600, 6400, 10), (4096, 4096, 5)])
def test_long_sides(b, rows, cols, steps, dtype):
    """X X^T's sums lose 3 k / 16 times 2^-25 on average (tolerance() has the derivation), 9.2e-5 at k = 16384, those of the other two 2.3e-5 each at 4096: 1.4e-4 < 2^-12.
    (Operands of 11 bits leave 4e-4 and more of what is beyond the rounding.)"""
    gen = torch.Generator(device="cuda")
    gen.manual_seed(rows + cols)
    x = torch.randn(rows, cols, generator=gen, device="cuda")
    want = x.double() if rows <= cols else x.double().t()
    want = want / want.norm()
    for _ in range(steps):
        a = want @ want.t()
        want = QUINTIC[0] * want + (QUINTIC[1] * a + QUINTIC[2] * (a @ a)) @ want
    want = want if rows <= cols else want.t()
    # (elements of some 2^-7, on which float16's subnormal numbers begin at 2^-14: brought near 1)
    scale = 2.0 ** round(float(-torch.log2(want.abs().mean())))
    got = b.orthogonalise(x, steps=steps, dtype=dtype, scale=scale).double()
    far = beyond_rounding(got.cpu().numpy(), (want * scale).cpu().numpy(), dtype)
    assert far <= 2.0 ** -12, far

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

"""Norms into 8-bit forms whose products h rstd weight reach the ends of fp32's range."""
import pytest
import torch

from oracle import f8_oracle as fo
from tests.test_gpu_f8 import DTYPES, KINDS, b, check_form, f64  # noqa: F401  (b: a fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("kind", KINDS)
def test_products_beyond_the_range_are_infinite(b, kind, dtype):
    """A single element of a row is 16 times its root's inverse: times 2^123 it is within the range, times 2^124 beyond it, and its block with it."""
    for cols in (256, 257):
        x = torch.zeros(3, cols, device="cuda")
        x[:, 5], x[1, 200] = 3.0, 1.0
        w = torch.full((cols,), 1.5, device="cuda")
        w[5] = 2.0 ** 123
        for bump in (1.0, 2.0):
            w[5] *= bump
            for forms in ("rows", "both"):
                out = b.rms_norm(x.to(dtype), w, 0.0, forms=forms, kind=kind)
                y = f64(x) * out.rstd.double().cpu().numpy()[:, None] * f64(w)
                y[abs(y) >= 2.0 ** 128] = float("inf")
                assert (abs(y[:, 5]) == float("inf")).sum() == (0 if bump == 1.0 else 2)
                check_form(out.y if forms == "rows" else out.y[0], y, kind)
                if forms == "both":
                    check_form(out.y[1], y.T.copy(), kind)
                v = b.f8_dequantise(out.y if forms == "rows" else out.y[0])
                assert torch.isnan(v[0, :128]).all() == (bump == 2.0) and torch.isfinite(v[:, 128:]).all()

"""The operators as a training step uses them: a layer's norm into 8 bits, its product and gradients, the exchange of the weight's gradient with error feedback, and
the orthogonalised update, against the same in 64 bits."""
import numpy as np
import pytest
import torch

from oracle import f8_oracle as fo
from tests.test_gpu_f8 import b, f64, matrix  # noqa: F401  (b: a fixture)

pytestmark = pytest.mark.gpu

TOKENS, IN, OUT, WORKERS = 260, 200, 328, 2


def values(form):
    return fo.decode(*fo.unpack(form.codes.cpu().numpy(), form.scales.cpu().numpy(), form.rows, form.cols), form.kind)


def far(got, want):
    return np.linalg.norm(f64(got) - want) / np.linalg.norm(want)


def test_a_layer_trains(b):
    ctx = b.ConEF([(OUT, IN, 1)], WORKERS, dict(kind="randk", k_num=1, k_den=2, seed=3), dict(kind="int8", block=256), 1.0)
    w, gain = matrix(OUT, IN, torch.float32, 1, 0.02), torch.ones(IN, device="cuda") * 1.25
    momentum = torch.zeros(OUT, IN, device="cuda")
    before = b.f8_timeouts()
    for t in range(2):
        grads = []
        w_rows, w_cols = b.f8_quantise(w, "both", square=True)
        for i in range(WORKERS):
            x, res, dy = (matrix(TOKENS, n, torch.bfloat16, 10 * t + 3 * i + j) for j, n in enumerate((IN, IN, OUT)))
            (n_rows, n_cols), h, rstd = b.rms_norm(x, gain, 1e-5, add=res, forms="both")
            y = b.f8_matmul(n_rows, w_rows)
            g_rows, g_cols = b.f8_quantise(dy, "both", kind="e5m2")
            dn = b.f8_matmul(g_rows, w_cols)
            dx, dgain = b.rms_norm_grad(dn, h, gain, rstd, add=res)
            dw = b.f8_matmul(g_cols, n_cols, dtype=torch.float32)
            grads.append(dw.view(-1))
            # in 64 bits, from the forms' values
            hh = (x.float() + res.float()).bfloat16()
            assert torch.equal(h, hh)
            assert far(y, values(n_rows) @ values(w_rows).T) <= 2.0 ** -8 + 1e-6
            assert far(dw, values(g_cols) @ values(n_cols).T) <= 1e-6
            want, want_gain = fo.rms_norm_grad(f64(dn), f64(h), f64(gain), rstd.cpu().numpy())
            assert far(dx, want + f64(res)) <= 2.0 ** -8 + 1e-5 and far(dgain, want_gain) <= 1e-5
            # ... and near the layer's own gradient: each 8-bit factor is off by half a step at most, 2^-4 (e4m3) and 2^-3 (e5m2) of its size
            n, _ = fo.rms_norm(f64(hh), f64(gain), 1e-5)
            assert far(dw, f64(dy).T @ n) <= 2.0 ** -4 + 2.0 ** -3 + 2.0 ** -7
        errors = [ctx.decompress_error(i).clone() for i in range(WORKERS)]
        ctx.step(t, grads)
        sums = {b.MSG_VALUES: ctx.reduce_messages(b.MSG_VALUES)}
        delta = torch.zeros(OUT * IN, device="cuda")
        ctx.apply_update(delta, sums)                       # minus the mean of what was sent
        assert int((delta != 0).sum()) <= OUT * IN // 2
        left = [ctx.decompress_error(i) for i in range(WORKERS)]
        # what was sent and what is kept are the gradients and what was kept before, but for int8's half a step
        kept = sum(f64(g) + f64(e) - f64(l) for g, e, l in zip(grads, errors, left)) / WORKERS
        assert np.abs(kept + f64(delta)).max() <= max(float(l.abs().max()) for l in left) / 127
        momentum.mul_(0.9).sub_(delta.view(OUT, IN))
        step = b.orthogonalise(momentum, scale=-0.02)
        assert far(step, fo.orthogonalise(f64(momentum), 5, (3.4445, -4.7750, 2.0315), -0.02)) <= 2.0 ** -8 + 5e-4
        w += step
    assert torch.isfinite(w).all() and ctx.last_status() == 0 and b.f8_timeouts() == before

"""A block of the mx4 state that is NaN: it stays so while an element of it is kept, and is finite after the step that sends the last ones, whichever kernels
run, also where it is a tensor's short last one."""
import numpy as np
import pytest
import torch

from tests import parity_util as pu
from tests.test_gpu_mx4_step import KINDS, compare, config

pytestmark = pytest.mark.gpu

# the last block has 1, 15, 16, 17, 31 and 32 elements, alone in its chunk or not
SIZES = [(1, 33, 1), (1, 47, 1), (3, 16, 1), (1, 49, 1), (1, 63, 1), (2, 32, 1), (1, 1, 0), (1, 513, 1), (7, 1000, 1), (1, 31, 1)]


def both(cfg):
    return [pu.make_gpu(cfg, fast=f) for f in (True, False)], pu.make_oracle(cfg)


def off_a_boundary(gd, shift):
    return [torch.cat([g.new_zeros(shift), g])[shift:] for g in gd] if shift else gd


def step(engines, o, cfg, t, gd, gh):
    from paper_2312_08538_b200 import binding as b
    with np.errstate(invalid="ignore"):
        res = o.step(t, gh)
    for eng in engines:
        out = eng.full_step(t, gd)
        assert np.array_equal(out[b.MSG_VALUES].cpu().numpy(), o.reduced(res, "values"), equal_nan=True)
        compare(eng, o, t)


@pytest.mark.parametrize("shift", [0, 1, 2, 3])
@pytest.mark.parametrize("q", [dict(kind="randk", k_num=1, k_den=1, seed=3), dict(kind="randblock", k_num=1, k_den=1, seed=3), dict(kind="identity")])
@pytest.mark.parametrize("kind", KINDS)
def test_all_of_it_is_sent(kind, q, shift):
    """The last block of every tensor is NaN before a step that sends everything."""
    cfg = config(kind, q, SIZES, 2)
    engines, o = both(cfg)
    for i in range(2):
        for l in o.compressed:
            o.state[i][l]["scales"][-1] = 255
            for eng in engines:
                eng.state(i, l)[1][-1] = 255
    gd, gh = pu.grads_both(cfg, 0)
    step(engines, o, cfg, 0, off_a_boundary(gd, shift), gh)
    for eng in engines:
        for i in range(2):
            assert not eng.decompress_error(i).any()         # (NaN counts)


@pytest.mark.parametrize("shift", [0, 1])
@pytest.mark.parametrize("q", [dict(kind="randk", k_num=1, k_den=2, seed=5), dict(kind="randblock", k_num=15, k_den=16, seed=5), dict(kind="randk", k_num=3, k_den=4, seed=7)])
@pytest.mark.parametrize("kind", KINDS)
def test_after_one_gradient_that_is_not_finite(kind, q, shift):
    """Blocks come back one by one, in the same step with all kernels and the oracle."""
    cfg = config(kind, q, SIZES, 2)
    engines, o = both(cfg)
    ends = np.cumsum([r * c for r, c, _ in SIZES])
    for t in range(12):
        gd, gh = pu.grads_both(cfg, t)
        if t == 0:
            for i, bad in enumerate((float("inf"), float("nan"))):
                for at in ends - 1:
                    gd[i][int(at)] = bad
                    gh[i][int(at)] = bad
        step(engines, o, cfg, t, off_a_boundary(gd, shift), gh)
    # (the block of one element that ends the first tensor has been sent by now)
    assert np.isfinite(o.decode(0, 0)).all() and np.isfinite(o.decode(1, 0)).all()


@pytest.mark.parametrize("fast", [True, False])
@pytest.mark.parametrize("kind", KINDS)
def test_a_job_clears_one_by_its_scale(kind, fast):
    cfg = config(kind, dict(kind="randk", k_num=1, k_den=100, seed=5), [(70, 33, 1)], 1)
    eng, o = pu.make_gpu(cfg, fast=fast), pu.make_oracle(cfg)
    for t in range(4):
        gd, gh = pu.grads_both(cfg, t)
        if t == 0:
            gd[0][100] = gh[0][100] = float("inf")
        with np.errstate(invalid="ignore"):
            o.step(t, gh)
        eng.full_step(t, gd)
        compare(eng, o, t)
        if t == 1:
            scales = eng.state(0, 0)[1]
            assert (scales == 255).sum() == 1
            scales[scales == 255] = 0
            o.state[0][0]["scales"][o.state[0][0]["scales"] == 255] = 0
            assert torch.isfinite(eng.decompress_error(0)).all()
    assert torch.isfinite(eng.decompress_error(0)).all()



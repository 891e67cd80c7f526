"""The step with its error state in microscaled 4-bit floats: indices, messages, codes and scales bit for bit those of the oracle."""
import numpy as np
import pytest
import torch

from oracle import mx4_oracle as mo
from paper_2312_08538_b200 import workloads as wl
from tests import parity_util as pu

pytestmark = pytest.mark.gpu

RAGGED = [(37, 53, 1), (19, 1, 0), (1, 7, 1), (64, 129, 1), (300, 1, 0), (5, 1000, 1), (1, 1, 0), (200, 96, 1), (3, 11, 1), (130, 257, 1), (70, 512, 1)]
KINDS = ["mx4", "mx4-stochastic"]


def config(kind, q, tensors=RAGGED, workers=3, **more):
    cfg = wl.config("tiny")
    cfg.update(tensors=tensors, n_workers=workers, q=q, c=dict(kind=kind, seed=4242, **more))
    return cfg


def state(eng, o, i, l):
    """(codes, scale bytes) of the library's state, and that nothing lies past the last element."""
    a, s = eng.state(i, l)
    raw, d = a.cpu().numpy(), o.d_of(l)
    codes = np.stack([raw & 15, raw >> 4], -1).reshape(-1)
    assert not codes[d:].any()
    return codes[:d], s.cpu().numpy()


def compare(eng, o, t):
    for i in range(o.N):
        for l in o.compressed:
            codes, scales = state(eng, o, i, l)
            st = o.state[i][l]
            assert np.array_equal(scales, st["scales"]), (t, i, l)
            assert np.array_equal(codes, st["codes"]), (t, i, l, np.argwhere(codes != st["codes"])[:3])
        assert np.array_equal(eng.decompress_error(i).cpu().numpy(), o.decompress_error(i), equal_nan=True)


def free_running(cfg, steps, fast=True, shift=0):
    from paper_2312_08538_b200 import binding as b
    eng, o = pu.make_gpu(cfg, fast=fast), pu.make_oracle(cfg)
    for t in range(steps):
        gd, gh = pu.grads_both(cfg, t)
        if shift:   # gradients off a 16-byte boundary
            gd = [torch.cat([g.new_zeros(shift), g])[shift:] for g in gd]
        res = o.step(t, gh)
        out = eng.full_step(t, gd)
        assert eng.last_status() == 0
        assert np.array_equal(out[b.MSG_VALUES].cpu().numpy(), o.reduced(res, "values"))
        if cfg["q"]["kind"] != "identity":
            for l in o.compressed:
                assert np.array_equal(eng.indices(l).cpu().numpy().view(np.uint32), res[l].idx)
        if o.reduced(res, "dense1d").size:
            assert np.array_equal(out[b.MSG_DENSE1D].cpu().numpy(), o.reduced(res, "dense1d"))
        compare(eng, o, t)
    return eng, o


@pytest.mark.parametrize("fast", [True, False])
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("q", [dict(kind="randk", k_num=3, k_den=100, seed=77), dict(kind="randblock", k_num=1, k_den=9, seed=8), dict(kind="identity"),
                               dict(kind="randk", k_num=1, k_den=2, seed=3)])
def test_bit_exact_over_steps(kind, q, fast):
    free_running(config(kind, q), 4, fast)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("beta", [0.5, 0.9])
def test_partial_error_feedback(kind, beta):
    free_running(config(kind, dict(kind="randk", k_num=3, k_den=100, seed=77), beta=beta), 3)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("shift", [1, 2, 3])
def test_gradients_off_a_boundary(kind, shift):
    free_running(config(kind, dict(kind="randk", k_num=1, k_den=30, seed=5), workers=2), 3, shift=shift)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("tensors,workers", [([(1, 33, 1)], 1), ([(1000, 1021, 1), (513, 1024, 1)], 2), ([(2, 2, 1)] * 40, 5)])
def test_other_models(kind, tensors, workers):
    free_running(config(kind, dict(kind="randk", k_num=1, k_den=100, seed=5), tensors, workers), 2)


@pytest.mark.parametrize("kind", KINDS)
def test_lowrank(kind):
    """Per step from the oracle's state and factors: the stored codes bit for bit, the factors within their tolerance."""
    from paper_2312_08538_b200 import binding as b
    cfg = wl.config("resnet50-mini")
    cfg["c"] = dict(kind=kind, seed=31)
    q0 = wl.q_init(cfg, "cuda")
    eng, o = pu.make_gpu(cfg, q_init=q0), pu.make_oracle(cfg, q_init=q0.cpu().numpy())
    for t in range(3):
        gd, gh = pu.grads_both(cfg, t)
        res = o.step(t, gh)
        eng.step(t, gd, 0)
        assert pu.frob_err(eng.reduce_messages(b.MSG_P).cpu().numpy(), o.reduced(res, "P")) <= pu.FROB
        for l in o.compressed:
            eng.factors(l, 0)["p_hat"].copy_(torch.from_numpy(res[l].Phat).cuda())
        eng.step(t, gd, 2)
        for l in o.compressed:
            for i in range(o.N):
                f = eng.factors(l, i)
                assert pu.frob_err(f["q_i"].cpu().numpy(), res[l].Qi[i]) <= pu.FROB
                f["q_i"].copy_(torch.from_numpy(res[l].Qi[i]).cuda())
        eng.step(t, gd, 3)
        assert np.array_equal(eng.reduce_messages(b.MSG_Q).cpu().numpy(), o.reduced(res, "Q"))
        compare(eng, o, t)


@pytest.mark.parametrize("fast", [True, False])
@pytest.mark.parametrize("kind", KINDS)
def test_a_residual_that_is_not_finite_takes_its_block(kind, fast):
    cfg = config(kind, dict(kind="randblock", k_num=1, k_den=50, seed=5), [(70, 33, 1), (9, 512, 1)], 2)
    eng, o = pu.make_gpu(cfg, fast=fast), pu.make_oracle(cfg)
    for t in range(2):
        gd, gh = pu.grads_both(cfg, t)
        if t == 0:
            for i, bad in enumerate((float("nan"), float("inf"))):
                for at in (40, 2309, 3000):
                    gd[i][at] = bad
                    gh[i][at] = bad
        with np.errstate(invalid="ignore"):
            o.step(t, gh)
        eng.full_step(t, gd)
        compare(eng, o, t)
    e = eng.decompress_error(0).cpu().numpy()
    assert np.isnan(e[32:64]).sum() >= 30 and np.isfinite(e[:32]).all() and np.isfinite(e[64:2304]).all()


@pytest.mark.parametrize("kind", KINDS)
def test_checkpoint_and_update(kind):
    cfg = config(kind, dict(kind="randk", k_num=1, k_den=10, seed=5), [(70, 33, 1), (5, 1, 0), (9, 512, 1)], 2)
    a = pu.make_gpu(cfg)
    for t in range(2):
        a.full_step(t, pu.grads_both(cfg, t)[0])
    c = pu.make_gpu(cfg)
    c.load_state_dict(a.state_dict())
    x, y = torch.zeros(70 * 33 + 5 + 9 * 512, device="cuda"), torch.zeros(70 * 33 + 5 + 9 * 512, device="cuda")
    for eng, v in ((a, x), (c, y)):
        eng.apply_update(v, eng.full_step(2, pu.grads_both(cfg, 2)[0]))
    assert torch.equal(x, y) and x.any()
    assert all(torch.equal(a.decompress_error(i), c.decompress_error(i)) for i in range(2))


def test_stochastic_state_is_that_of_a_quantised_row():
    """The step's numbers are those of the quantisation of one row: its code for the same values, worker, tensor and step."""
    from paper_2312_08538_b200 import binding as b
    cfg = config("mx4-stochastic", dict(kind="randblock", k_num=1, k_den=10 ** 6, seed=5), [(3, 7, 0), (10, 333, 1)], 2)
    cfg["lr"] = 1.0
    eng = pu.make_gpu(cfg)
    gd, _ = pu.grads_both(cfg, 6)
    eng.full_step(6, gd)
    at = int(eng.indices(1)[0])
    for i in range(2):
        g = gd[i][21:].clone()
        g[at] = 0.0
        want = b.mx4_dequantise(b.mx4_quantise(g, stochastic=True, draw=b.Draw(4242, i, 1, 6)))
        assert torch.equal(eng.decompress_error(i), want.view(-1))

"""The plain statement of the microscaled 4-bit floats and counter-based draws against definitions worked out another way, and what
the library's calls on them refuse on the host."""
import ctypes as C
import math
from fractions import Fraction

import numpy as np
import pytest

from oracle import mx4_oracle as mo


def _one(x, u=None):
    """Brute force over the eight values and all exponents, in rational numbers: (codes, scale byte) of one block."""
    if not all(math.isfinite(v) for v in x):
        return [0] * len(x), mo.NAN_SCALE
    e = next(e for e in range(-127, 128) if max(abs(Fraction(v)) for v in x) <= 6 * Fraction(2) ** e)
    codes = []
    for i, v in enumerate(x):
        y = abs(Fraction(v)) / Fraction(2) ** e
        grid = [Fraction(g) for g in mo.GRID]
        if u is None:
            best = min(abs(y - g) for g in grid)
            near = [c for c in range(8) if abs(y - grid[c]) == best]
            c = near[0] if len(near) == 1 else next(c for c in near if c % 2 == 0)
        else:
            low = max(c for c in range(7) if grid[c] <= y)
            f = (y - grid[low]) / (grid[low + 1] - grid[low])
            c = low + (math.floor(f * 65536 + Fraction(1, 2)) + int(u[i]) >= 65536)
        codes.append(c + (8 if math.copysign(1.0, v) < 0 else 0))
    return codes, e + 127


def _blocks():
    rng = np.random.default_rng(5)
    yield np.zeros(32)
    yield np.array([0.25, -0.75, 1.25, -1.75, 2.5, 3.5, 5.0, 6.0, -0.0, 0.2500001, 4.9999995] + [0.0] * 21)     # ties
    yield np.array([6.0000005] + [1.0] * 31)
    yield np.array([1.5, -1.5000001])
    yield np.array([3.4028235e38, 1e-45, -1e30])
    yield np.array([1e-45, -1e-45, 3e-45])
    yield np.array([float("inf"), 1.0])
    yield np.array([float("nan"), 1.0, 2.0])
    for _ in range(60):
        yield (rng.standard_normal(32) * 2.0 ** rng.integers(-140, 120)).astype(np.float32).astype(np.float64)


@pytest.mark.parametrize("stochastic", [False, True])
def test_codes_and_scales_by_brute_force(stochastic):
    rng = np.random.default_rng(6)
    for x in _blocks():
        u = rng.integers(0, 65536, x.size) if stochastic else None
        codes, scales = mo.encode(x[None], None if u is None else u[None])
        want, scale = _one([float(v) for v in x], u)
        assert codes[0].tolist() == want and scales.tolist() == [[scale]]


def test_rounding_extremes():
    x = np.array([[6.0, 0.25, 1.1, 4.5, 5.9999995, 2.0]])
    assert mo.encode(x, np.zeros((1, 6), np.int64))[0].tolist() == [[7, 0, 2, 6, 7, 4]]         # (1 - f < 2^-17 always goes up)
    assert mo.encode(x, np.full((1, 6), 65535))[0].tolist() == [[7, 1, 3, 7, 7, 4]]


def test_stochastic_rounding_is_unbiased_to_2_to_minus_17():
    """Over all 65536 numbers the mean is the value, but for 2^-17 of a step at most."""
    u = np.arange(65536)[:, None]
    for v in (0.1, 0.49, 0.7, 1.3, 2.2, 3.9, 5.3):
        x = np.full((65536, 2), v)
        x[:, 1] = 6.0
        mean = mo.decode(*mo.encode(x, np.concatenate([u, u], 1)))[:, 0].mean()
        step = 0.5 if v < 2 else 1.0 if v < 4 else 2.0
        assert abs(mean - v) <= step * 2.0 ** -17 + 1e-12


@pytest.mark.parametrize("rows,cols", [(1, 1), (3, 33), (130, 129), (5, 257), (257, 31)])
def test_packing_there_and_back(rows, cols):
    rng = np.random.default_rng(7)
    codes = rng.integers(0, 16, (rows, cols)).astype(np.uint8)
    scales = rng.integers(0, 256, (rows, (cols + 31) // 32)).astype(np.uint8)
    a, b = mo.unpack(*mo.pack(codes, scales), rows, cols)
    assert np.array_equal(a, codes) and np.array_equal(b, scales)


def test_numbers_are_the_hash_of_the_step_oracle():
    from oracle import conef_oracle as orc
    got = mo.numbers(11, 2, 3, 4, 5, 7, mo.ROUNDING)
    for r in range(5):
        for c in range(7):
            word = orc.h64(orc.mix64(11 + 2 + 1), 3, 4, 2 * (r * 2 + c // 4) + 1)
            assert got[r, c] == (word >> (16 * (c % 4))) & 0xFFFF


def test_numbers_look_uniform_and_differ_between_draws():
    a = mo.numbers(1, 0, 0, 0, 400, 500, mo.DROPOUT)
    n, hist = a.size, np.bincount(a.ravel() >> 8, minlength=256)
    # each of 256 bins: mean n/256, standard deviation sqrt(n/256); six of those either way
    assert np.abs(hist - n / 256).max() <= 6 * math.sqrt(n / 256)
    for other in ((2, 0, 0, 0), (1, 1, 0, 0), (1, 0, 1, 0), (1, 0, 0, 1)):
        same = (mo.numbers(*other, 400, 500, mo.DROPOUT) == a).mean()
        assert same <= 1 / 65536 + 6 * math.sqrt(1 / 65536 / n)


def test_oracle_step_conserves_what_it_sends_and_keeps():
    """delta + decoded error is p but for the rounding: half a step of the block's scale at most."""
    from oracle import conef_oracle as orc
    for kind, part in (("mx4", 0.5), ("mx4-stochastic", 1.0)):
        o = orc.ConEFOracle([(9, 37, 1)], 1, orc.QCfg(kind="randk", k_num=1, k_den=10, seed=3), orc.CCfg(kind=kind, seed=9), 0.5)
        g = np.random.default_rng(2).standard_normal(9 * 37).astype(np.float32)
        res = o.step(0, [g], record=True)[0]
        e = o.decompress_error(0)
        assert not e[res.idx].any()
        scale = np.repeat(np.ldexp(1.0, o.state[0][0]["scales"].astype(int) - 127), 32)[:g.size]
        assert (np.abs(e - res.r[0]) <= 2 * part * scale).all()        # (the widest step is 2)


# ------------------------------------------------------------------ refusals (nothing is launched)

@pytest.fixture(scope="module")
def b():
    from paper_2312_08538_b200 import build
    build.build_library()
    from paper_2312_08538_b200 import binding
    return binding


P = 1 << 20   # an address that no call here reaches


def test_dropout_refusals(b):
    ok = dict(x=P, add=None, out=P, dtype=b.F32, rows=2, cols=8, ld=8, add_ld=8, out_ld=8, p=0.5, draw=C.byref(b.Draw(1, 0, 0, 0)), stream=None)

    def rc(**kw):
        return b.lib.conef_dropout(*{**ok, **kw}.values())

    for kw in (dict(dtype=3), dict(rows=-1), dict(cols=-1), dict(ld=7), dict(out_ld=7), dict(x=None), dict(out=None), dict(x=P + 2), dict(add=P + 1),
               dict(p=-0.1), dict(p=1.1), dict(p=float("nan")), dict(draw=None), dict(draw=C.byref(b.Draw(1, -1, 0, 0))),
               dict(draw=C.byref(b.Draw(1, 0, 0, -1))), dict(draw=C.byref(b.Draw(1, 0, -2, 0)))):
        assert rc(**kw) == b.ERR_INVALID_ARG, kw
    for kw in (dict(rows=1 << 31), dict(cols=1 << 31, ld=1 << 31), dict(out_ld=1 << 31)):
        assert rc(**kw) == b.ERR_UNSUPPORTED, kw
    assert rc(rows=0) == b.OK and rc(cols=0) == b.OK


def test_quantise_refusals(b):
    ok = dict(x=P, dtype=b.BF16, rows=2, cols=8, ld=8, p=0.0, stochastic=0, draw=None, codes=P, scales=P, codes_t=None, scales_t=None, stream=None)

    def rc(**kw):
        return b.lib.conef_mx4_quantise(*{**ok, **kw}.values())

    for kw in (dict(dtype=-1), dict(ld=3), dict(x=P + 1), dict(x=None), dict(p=2.0), dict(p=0.5), dict(stochastic=1), dict(codes=None), dict(scales=None),
               dict(codes=None, scales=None), dict(codes_t=P), dict(scales_t=P), dict(codes=P + 8), dict(scales=P + 4), dict(rows=-3)):
        assert rc(**kw) == b.ERR_INVALID_ARG, kw
    assert rc(rows=1 << 31) == b.ERR_UNSUPPORTED
    assert rc(rows=0) == b.OK and rc(cols=0) == b.OK


def test_dequantise_and_product_refusals(b):
    ok = dict(codes=P, scales=P, rows=2, cols=8, out=P, dtype=b.F32, ld=8, stream=None)

    def rc(**kw):
        return b.lib.conef_mx4_dequantise(*{**ok, **kw}.values())

    for kw in (dict(codes=None), dict(scales=None), dict(codes=P + 1), dict(out=None), dict(ld=7), dict(dtype=9), dict(rows=-1)):
        assert rc(**kw) == b.ERR_INVALID_ARG, kw
    assert rc(rows=0) == b.OK
    ok = dict(a=P, sa=P, m=2, b=P, sb=P, n=3, k=8, out=P, dtype=b.F16, ld=3, stream=None)

    def rc(**kw):   # noqa: F811
        return b.lib.conef_mx4_matmul(*{**ok, **kw}.values())

    for kw in (dict(a=None), dict(sb=None), dict(b=P + 4), dict(out=P + 1), dict(ld=2), dict(dtype=3), dict(k=-1), dict(m=-1), dict(n=-1)):
        assert rc(**kw) == b.ERR_INVALID_ARG, kw
    assert rc(k=1 << 31) == b.ERR_UNSUPPORTED
    assert rc(m=0) == b.OK and rc(n=0, ld=0) == b.OK


def test_sizes(b):
    c, s = C.c_size_t(), C.c_size_t()
    for rows, cols in ((0, 5), (1, 1), (128, 128), (129, 4097), (50257, 1600)):
        assert b.lib.conef_mx4_bytes(rows, cols, C.byref(c), C.byref(s)) == b.OK
        assert (c.value, s.value) == b._mx4_sizes(rows, cols)
    assert b.lib.conef_mx4_bytes(-1, 4, None, None) == b.ERR_INVALID_ARG
    assert b.lib.conef_mx4_bytes(4, 1 << 31, None, None) == b.ERR_UNSUPPORTED


def test_the_binding_refuses_what_is_not_on_a_gpu(b):
    import torch
    x = torch.zeros(4, 8)
    form = b.MX4(4, 8, torch.zeros(64, dtype=torch.uint8), torch.zeros(512, dtype=torch.uint8))
    for call in (lambda: b.dropout(x, 0.5, b.Draw(1, 0, 0, 0)), lambda: b.mx4_quantise(x), lambda: b.mx4_dequantise(form), lambda: b.mx4_matmul(form, form)):
        with pytest.raises(b.ConEFError) as e:
            call()
        assert e.value.code == b.ERR_INVALID_ARG


def test_configurations_of_the_step(b):
    q = dict(kind="randk", k_num=1, k_den=10, seed=1)
    d = 1600 * 6400
    for kind in ("mx4", "mx4-stochastic"):
        mx = b.conef_workspace_bytes([(1600, 6400, 1)], 1, q, dict(kind=kind))
        dense = b.conef_workspace_bytes([(1600, 6400, 1)], 1, q, dict(kind="identity"))
        assert dense - mx == pytest.approx(d * (4 - 0.5 - 1 / 32), abs=4096)
        for bad in (dict(iconef=1), dict(iconef=2)):
            with pytest.raises(b.ConEFError) as e:
                b.conef_workspace_bytes([(4, 5, 1)], 2, q, dict(kind=kind, **bad))
            assert e.value.code == b.ERR_UNSUPPORTED
    t, qc, cc, n = b.make_tensors([(4, 5, 1)]), b.make_q(q, None), b.make_c(dict(kind="mx4")), C.c_size_t()
    cc.kind = 8
    assert b.lib.conef_workspace_bytes(t, 1, 1, C.byref(qc), C.byref(cc), C.byref(n)) == b.ERR_INVALID_ARG

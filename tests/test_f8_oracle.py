"""The plain statement of 8-bit floats, norms and orthogonalised updates against brute force and differences; refusals of the operators (nothing is launched)."""
import ctypes as C
from fractions import Fraction

import numpy as np
import pytest

from oracle import f8_oracle as fo

KINDS = ["e4m3", "e5m2"]
QUINTIC = (3.4445, -4.7750, 2.0315)


@pytest.mark.parametrize("kind", KINDS)
def test_values_of_the_types(kind):
    import torch
    t = {"e4m3": torch.float8_e4m3fn, "e5m2": torch.float8_e5m2}[kind]
    v = torch.arange(128, dtype=torch.uint8).view(t).double().numpy()
    g = fo.grid(kind)
    assert np.array_equal(g, v[:g.size]) and not np.isfinite(v[g.size:]).any()


def brute(v, e, kind):
    """The code of v 2^-e by search in rational numbers, to nearest, ties to the even code."""
    y = Fraction(abs(v)) / Fraction(2) ** int(e)
    far = [abs(Fraction(float(g)) - y) for g in fo.grid(kind)]
    best = min(far)
    at = [i for i, f in enumerate(far) if f == best]
    code = at[0] if len(at) == 1 or at[0] % 2 == 0 else at[1]
    return code + (128 if np.signbit(v) else 0)


@pytest.mark.parametrize("kind", KINDS)
def test_encode_against_brute_force(kind):
    gen = np.random.default_rng(3)
    g = fo.grid(kind)
    ties = np.concatenate([(g[:-1] + g[1:]) / 2, g])
    for scale in (1.0, 2.0 ** -130, 2.0 ** 100, 0.37):
        x = np.concatenate([gen.standard_normal(60) * np.exp2(gen.integers(-12, 8, 60)), ties[gen.integers(0, ties.size, 40)], [0.0, -0.0, g[-1]]]) * scale
        x = x.astype(np.float32).astype(np.float64)[None]
        codes, scales = fo.encode(x, kind)
        e = int(scales[0, 0]) - 127
        assert np.abs(x).max() <= g[-1] * 2.0 ** e and (e == -127 or np.abs(x).max() > g[-1] * 2.0 ** (e - 1))
        assert codes[0].tolist() == [brute(v, e, kind) for v in x[0]]
        back = fo.decode(codes, scales, kind)
        assert (np.abs(back - x) <= np.maximum(np.abs(x) * 2.0 ** (-4 if kind == "e4m3" else -3), g[1] * 2.0 ** e / 2)).all()


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("rows,cols", [(1, 1), (3, 130), (129, 513), (300, 127)])
def test_pack_and_unpack(kind, rows, cols):
    x = np.random.default_rng(rows).standard_normal((rows, cols))
    codes, scales = fo.encode(x, kind)
    c, s = fo.unpack(*fo.pack(codes, scales), rows, cols)
    assert np.array_equal(c, codes) and np.array_equal(s, scales)


@pytest.mark.parametrize("kind", KINDS)
def test_square_blocks_have_one_scale_and_transpose(kind):
    x = np.random.default_rng(1).standard_normal((300, 270)) * np.exp2(np.random.default_rng(2).integers(-9, 9, (300, 270)))
    codes, scales = fo.encode(x, kind, True)
    codes_t, scales_t = fo.encode(x.T.copy(), kind, True)
    assert np.array_equal(codes, codes_t.T)
    for r in range(0, 300, 128):
        assert (scales[r:r + 128] == scales[r]).all()
    assert np.array_equal(scales[::128], scales_t[::128].T)


@pytest.mark.parametrize("kind", KINDS)
def test_blocks_with_infinities_and_nan(kind):
    x = np.ones((3, 260))
    x[0, 5], x[1, 129], x[2, 259] = np.inf, np.nan, -np.inf
    codes, scales = fo.encode(x, kind)
    assert scales[0, 0] == scales[1, 1] == scales[2, 2] == 255 and (scales == 255).sum() == 3
    assert not codes[0, :128].any() and np.isnan(fo.decode(codes, scales, kind)[0, :128]).all()


def test_norm_gradient_against_differences():
    gen = np.random.default_rng(5)
    h, dy, w = gen.standard_normal((4, 37)), gen.standard_normal((4, 37)), gen.standard_normal(37)
    eps = 0.1

    def loss(h, w):
        return (dy * (h / np.sqrt((h * h).mean(1, keepdims=True) + eps) * w)).sum()

    r = 1.0 / np.sqrt((h * h).mean(1) + eps)
    dx, dw = fo.rms_norm_grad(dy, h, w, r)
    step = 1e-6
    for i, j in ((0, 0), (1, 5), (3, 36)):
        d = np.zeros_like(h)
        d[i, j] = step
        assert (loss(h + d, w) - loss(h - d, w)) / (2 * step) == pytest.approx(dx[i, j], abs=1e-8)
    for j in (0, 20):
        d = np.zeros_like(w)
        d[j] = step
        assert (loss(h, w + d) - loss(h, w - d)) / (2 * step) == pytest.approx(dw[j], abs=1e-8)


@pytest.mark.parametrize("rows,cols", [(5, 9), (9, 5), (6, 6), (1, 4)])
def test_orthogonalise_is_the_polynomial_of_the_singular_values(rows, cols):
    x = np.random.default_rng(rows * cols).standard_normal((rows, cols))
    u, s, v = np.linalg.svd(x, full_matrices=False)
    s = s / np.sqrt((s * s).sum())
    a, b, c = QUINTIC
    for _ in range(4):
        s = a * s + b * s ** 3 + c * s ** 5
    assert np.allclose(fo.orthogonalise(x, 4, QUINTIC, 0.5), 0.5 * (u * s) @ v, atol=1e-10)
    assert not fo.orthogonalise(np.zeros((rows, cols)), 5, QUINTIC).any()


# ------------------------------------------------------------------ refusals (nothing is launched)

@pytest.fixture(scope="module")
def b():
    from paper_2312_08538_b200 import build
    build.build_library()
    from paper_2312_08538_b200 import binding
    return binding


P = 1 << 20   # an address that no call here reaches


def refuses(b, name, ok, bad, unsupported=(), fine=(), small=()):
    call = getattr(b.lib, name)
    for cases, code in ((bad, b.ERR_INVALID_ARG), (unsupported, b.ERR_UNSUPPORTED), (fine, b.OK), (small, b.ERR_WORKSPACE_TOO_SMALL)):
        for kw in cases:
            assert set(kw) <= set(ok), kw
            assert call(*{**ok, **kw}.values()) == code, kw


def test_quantise_refusals(b):
    ok = dict(x=P, dtype=b.BF16, rows=2, cols=8, ld=8, kind=b.E4M3, square=0, codes=P, scales=P, codes_t=None, scales_t=None, stream=None)
    refuses(b, "conef_f8_quantise", ok,
            (dict(dtype=-1), dict(ld=3), dict(x=P + 1), dict(x=None), dict(kind=2), dict(kind=-1), dict(codes=None), dict(scales=None), dict(codes=None, scales=None),
             dict(codes_t=P), dict(scales_t=P), dict(codes=P + 8), dict(scales=P + 4), dict(rows=-3)),
            (dict(rows=1 << 31), dict(cols=1 << 31, ld=1 << 31), dict(rows=(1 << 31) - 1, cols=1 << 14, ld=1 << 14, codes_t=P, scales_t=P)), (dict(rows=0), dict(cols=0)))


def test_dequantise_and_product_refusals(b):
    ok = dict(codes=P, scales=P, rows=2, cols=8, kind=b.E5M2, out=P, dtype=b.F32, ld=8, stream=None)
    refuses(b, "conef_f8_dequantise", ok, (dict(codes=None), dict(scales=None), dict(codes=P + 1), dict(out=None), dict(ld=7), dict(dtype=9), dict(rows=-1), dict(kind=7)),
            (dict(rows=1 << 31),), (dict(rows=0), dict(cols=0)))
    ok = dict(a=P, sa=P, ka=b.E4M3, m=2, b=P, sb=P, kb=b.E5M2, n=3, k=8, out=P, dtype=b.F16, ld=3, stream=None)
    refuses(b, "conef_f8_matmul", ok, (dict(a=None), dict(sb=None), dict(b=P + 4), dict(out=P + 1), dict(ld=2), dict(dtype=3), dict(k=-1), dict(m=-1), dict(n=-1), dict(ka=2),
                                       dict(kb=-1)), (dict(k=1 << 31),), (dict(m=0), dict(n=0, ld=0)))


def test_norm_refusals(b):
    ok = dict(x=P, add=P, w=P, dtype=b.BF16, w_dtype=b.F32, rows=2, cols=8, x_ld=8, add_ld=8, eps=1e-5, h=P, h_ld=8, rstd=P, y=P, y_ld=8, kind=0, codes=None, scales=None,
              codes_t=None, scales_t=None, stream=None)
    refuses(b, "conef_rms_norm", ok,
            (dict(x=None), dict(w=None), dict(h=None), dict(rstd=None), dict(add=None), dict(x=P + 1), dict(w=P + 2), dict(rstd=P + 2), dict(y=P + 1), dict(w_dtype=b.F16),
             dict(dtype=b.F32, w_dtype=b.BF16), dict(eps=-1.0), dict(eps=float("nan")), dict(eps=float("inf")), dict(codes=P, scales=P), dict(y=None, codes=P),
             dict(y=None, codes_t=P), dict(y=None, codes=P, scales=P, kind=2), dict(y=None, codes=P + 8, scales=P), dict(h_ld=7), dict(y_ld=7), dict(add_ld=7), dict(rows=-1)),
            (dict(rows=1 << 31),), (dict(rows=0), dict(cols=0, x_ld=0, add_ld=0, h_ld=0, y_ld=0)))
    ok = dict(dy=P, h=P, w=P, rstd=P, add=P, dtype=b.F16, w_dtype=b.F16, rows=2, cols=8, dy_ld=8, h_ld=8, add_ld=8, dx=P, dx_ld=8, dw=P, ws=P, bytes=1 << 20, stream=None)
    refuses(b, "conef_rms_norm_grad", ok,
            (dict(dy=None), dict(h=None), dict(w=None), dict(rstd=None), dict(dx=None), dict(add=P + 1), dict(ws=P + 2), dict(dw=P + 1), dict(dx_ld=7), dict(w_dtype=b.BF16)),
            (dict(rows=1 << 31),), (dict(rows=0, dw=None), dict(cols=0, dy_ld=0, h_ld=0, add_ld=0, dx_ld=0)), (dict(ws=None), dict(bytes=31)))


def test_orthogonalise_refusals(b):
    good = (C.c_double * 3)(*QUINTIC)
    ok = dict(x=P, dtype=b.F32, batch=2, rows=4, cols=8, ld=8, stride=32, steps=5, c=good, scale=1.0, out=P, out_dtype=b.BF16, out_ld=8, out_stride=32, ws=P, bytes=1 << 20,
              stream=None)
    refuses(b, "conef_orthogonalise", ok,
            (dict(x=None), dict(out=None), dict(x=P + 2), dict(ld=7), dict(stride=31), dict(out_stride=30), dict(out_dtype=b.F32), dict(out_dtype=3), dict(steps=0), dict(steps=33),
             dict(c=None), dict(c=(C.c_double * 3)(30.0, 0.0, 0.0)), dict(c=(C.c_double * 3)(float("nan"), 0.0, 0.0)), dict(scale=float("inf")), dict(batch=-1), dict(rows=-1),
             dict(ws=P + 64)),
            (dict(batch=1 << 16), dict(rows=1 << 31)), (dict(batch=0), dict(rows=0), dict(cols=0, ld=0, out_ld=0)), (dict(ws=None), dict(bytes=1000)))


def test_sizes(b):
    c, s = C.c_size_t(), C.c_size_t()
    for rows, cols in ((0, 5), (1, 1), (128, 128), (129, 4097), (50257, 1600)):
        assert b.lib.conef_f8_bytes(rows, cols, C.byref(c), C.byref(s)) == b.OK
        assert (c.value, s.value) == b._f8_sizes(rows, cols)
    assert b.lib.conef_f8_bytes(-1, 4, None, None) == b.ERR_INVALID_ARG
    assert b.lib.conef_f8_bytes(4, 1 << 31, None, None) == b.ERR_UNSUPPORTED
    assert b.lib.conef_rms_norm_grad_bytes(8, -1, C.byref(c)) == b.ERR_INVALID_ARG
    assert b.lib.conef_orthogonalise_bytes(1, 4, 4, None) == b.ERR_INVALID_ARG
    assert b.lib.conef_orthogonalise_bytes(1, 70, 130, C.byref(c)) == b.OK and c.value >= 70 * (2 * 192 + 2 * 128) * 4


def test_the_binding_refuses_what_is_not_on_a_gpu(b):
    import torch
    x, w, r = torch.zeros(4, 8), torch.zeros(8), torch.zeros(4)
    form = b.F8(4, 8, "e4m3", torch.zeros(512, dtype=torch.uint8), torch.zeros(512, dtype=torch.uint8))
    for call in (lambda: b.f8_quantise(x), lambda: b.f8_dequantise(form), lambda: b.f8_matmul(form, form), lambda: b.rms_norm(x, w), lambda: b.rms_norm_grad(x, x, w, r),
                 lambda: b.orthogonalise(x), lambda: b.orthogonalise(w), lambda: b.orthogonalise(x, dtype=torch.float32)):
        with pytest.raises(b.ConEFError) as e:
            call()
        assert e.value.code == b.ERR_INVALID_ARG

"""Dropout, quantisation to microscaled 4-bit floats, and their products against the plain statement in 64 bits."""
import numpy as np
import pytest
import torch

from oracle import mx4_oracle as mo

pytestmark = pytest.mark.gpu

EPS = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}   # half a step, relative
TINY = {torch.float32: 2.0 ** -149, torch.bfloat16: 2.0 ** -133, torch.float16: 2.0 ** -24}
DTYPES = [torch.float32, torch.bfloat16, torch.float16]
SEED = (77, 1, 5, 9)


@pytest.fixture(scope="module")
def b():
    from paper_2312_08538_b200 import binding
    return binding


def draw(b):
    return b.Draw(*SEED)


def matrix(rows, cols, dtype, seed=0, scale=1.0):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(1000 * rows + cols + seed)
    x = torch.randn(rows, cols, generator=gen, device="cuda")
    x *= torch.exp2(torch.randn(1, cols, generator=gen, device="cuda") * 2) * scale
    return x.to(dtype)


def f64(t):
    return t.double().cpu().numpy()


def strided(x, front=3, behind=2):
    """The same matrix as columns of a wider one, and that one."""
    wide = torch.full((x.shape[0], x.shape[1] + front + behind), 7.0, dtype=x.dtype, device="cuda")
    view = wide[:, front:front + x.shape[1]]
    view.copy_(x)
    return view, wide


# ------------------------------------------------------------------ dropout

def check_dropout(y, x, p, add=None, numbers=SEED):
    """One rounding of the scale to fp32, one of product plus sum, one to the type."""
    rows, cols = x.shape
    u = mo.numbers(*numbers, rows, cols, mo.DROPOUT)
    with np.errstate(invalid="ignore"):
        kept = mo.dropout(f64(x), p, u)
        want = kept + (0.0 if add is None else f64(add))
    tol = np.abs(kept) * 2.0 ** -24 * 1.001 + np.abs(want) * (2.0 ** -24 + EPS[x.dtype]) * 1.001 + TINY[x.dtype]
    got = f64(y)
    assert got.shape == want.shape
    off = ~(np.abs(got - want) <= tol) & ~((got == want) | (np.isnan(got) & np.isnan(want)))
    assert not off.any(), (np.argwhere(off)[:3], got[off][:3], want[off][:3])
    if add is None:
        assert (got[u < round(p * 65536)] == 0).all()


SHAPES = [(1, 1), (1, 3), (2, 4), (1, 1600), (7, 1600), (5, 33), (64, 31), (3, 127), (33, 1301), (2, 8192), (300, 8), (1000, 2), (70, 250), (1, 100003), (130, 4097)]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows,cols", SHAPES)
def test_dropout(b, rows, cols, dtype):
    x, r = matrix(rows, cols, dtype), matrix(rows, cols, dtype, 1)
    for p in (0.1, 0.731):
        check_dropout(b.dropout(x, p, draw(b)), x, p)
        check_dropout(b.dropout(x, p, draw(b), add=r), x, p, r)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("p", [0.0, 2.0 ** -16, 0.5, 1 - 2.0 ** -16, 1.0, 2.0 ** -18])
def test_dropout_probabilities(b, dtype, p):
    x, r = matrix(37, 203, dtype), matrix(37, 203, dtype, 1)
    y = b.dropout(x, p, draw(b))
    check_dropout(y, x, p)
    check_dropout(b.dropout(x, p, draw(b), add=r), x, p, r)
    if round(p * 65536) == 0:
        assert torch.equal(y, x)
    if p == 1.0:
        assert not y.any() and torch.equal(b.dropout(x, p, draw(b), add=r), r)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("front", [0, 1, 2, 3, 4, 5, 7, 8])
@pytest.mark.parametrize("rows,cols", [(9, 1301), (9, 64), (17, 5), (3, 1024)])
def test_dropout_of_strided_rows_leaves_what_lies_between(b, dtype, front, rows, cols):
    x, r = matrix(rows, cols, dtype), matrix(rows, cols, dtype, 1)
    xs, _ = strided(x, front, 3)
    rs, _ = strided(r, front, 3)
    other, wide = strided(x, front, 3)
    got = b.dropout(xs, 0.3, draw(b), add=rs, out=other)
    assert got is other
    check_dropout(got, x, 0.3, r)
    assert (wide[:, :front] == 7).all() and (wide[:, front + cols:] == 7).all()
    check_dropout(b.dropout(xs, 0.3, draw(b)), x, 0.3)                                   # (rows of x and of the result start on different boundaries)
    check_dropout(b.dropout(x, 0.3, draw(b), add=rs), x, 0.3, r)


@pytest.mark.parametrize("dtype", DTYPES)
def test_dropout_in_place_and_into_the_residual(b, dtype):
    for shape in ((33, 1301), (8, 1600)):
        x, r = matrix(*shape, dtype), matrix(*shape, dtype, 1)
        want = b.dropout(x, 0.4, draw(b), add=r)
        x1, r1 = x.clone(), r.clone()
        b.dropout(x1, 0.4, draw(b), add=r, out=x1)
        b.dropout(x, 0.4, draw(b), add=r1, out=r1)
        assert torch.equal(x1, want) and torch.equal(r1, want)
        y = b.dropout(x, 0.4, draw(b))
        x2 = x.clone()
        b.dropout(x2, 0.4, draw(b), out=x2)
        assert torch.equal(x2, y)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("front", [1, 2, 3, 5, 7])
@pytest.mark.parametrize("rows,cols", [(40, 33), (3, 1301), (200, 5), (50, 2), (9, 64), (1, 1000), (2000, 130)])
def test_dropout_of_arrays_that_begin_off_a_boundary(b, dtype, front, rows, cols):
    x, r = matrix(rows, cols, dtype), matrix(rows, cols, dtype, 1)

    def moved(t, by):
        whole = torch.full((t.numel() + by + 9,), 7.0, dtype=dtype, device="cuda")
        whole[by:by + t.numel()] = t.reshape(-1)
        return whole[by:by + t.numel()].view(rows, cols), whole

    (xs, _), (rs, _), (ys, whole) = moved(x, front), moved(r, front), moved(x, front)
    check_dropout(b.dropout(xs, 0.3, draw(b), add=rs, out=ys), x, 0.3, r)
    assert (whole[:front] == 7).all() and (whole[front + rows * cols:] == 7).all()
    check_dropout(b.dropout(xs, 0.3, draw(b), out=ys), x, 0.3)
    assert (whole[:front] == 7).all() and (whole[front + rows * cols:] == 7).all()
    check_dropout(b.dropout(xs, 0.3, draw(b), add=r), x, 0.3, r)       # (each off by something else)


def test_dropout_takes_any_leading_dimensions(b):
    x = matrix(24, 50, torch.bfloat16)
    want = b.dropout(x, 0.2, draw(b))
    assert torch.equal(b.dropout(x.view(2, 3, 4, 50), 0.2, draw(b)).view(24, 50), want)
    assert torch.equal(b.dropout(x.view(1, 24, 1, 50), 0.2, draw(b)).view(24, 50), want)
    assert torch.equal(b.dropout(x[3], 0.2, draw(b)), b.dropout(x[3:4], 0.2, draw(b))[0])
    for shape in ((0, 5), (5, 0), (0,), (2, 0, 3)):
        e = torch.empty(shape, device="cuda")
        assert b.dropout(e, 0.5, draw(b)).shape == e.shape
    for bad in (x.t(), x.view(4, 6, 50).transpose(0, 1), x.expand(2, 24, 50), x[:, ::2], x.double(), torch.tensor(1.0, device="cuda")):
        with pytest.raises(b.ConEFError):
            b.dropout(bad, 0.5, draw(b))
    with pytest.raises(b.ConEFError):
        b.dropout(x, 0.5, draw(b), add=x.float())
    with pytest.raises(b.ConEFError):
        b.dropout(x, 0.5, draw(b), add=x[:, :49])
    with pytest.raises(b.ConEFError):
        b.dropout(x, 0.5, None)


def test_dropout_of_values_that_are_not_finite(b):
    """A dropped element leaves no trace, be it NaN; a kept one is as IEEE says."""
    x = matrix(40, 301, torch.float32)
    x[::3, ::5] = float("nan")
    x[1::3, ::5] = float("inf")
    r = matrix(40, 301, torch.float32, 1)
    u = mo.numbers(*SEED, 40, 301, mo.DROPOUT)
    for add in (None, r):
        y = f64(b.dropout(x, 0.5, draw(b), add=add))
        gone = u < 32768
        assert (y[gone] == (0.0 if add is None else f64(r)[gone])).all()
        want = f64(x)[~gone] * 2 + (0.0 if add is None else f64(r)[~gone])
        fine = np.isfinite(want)
        assert np.array_equal(np.isnan(y[~gone]), np.isnan(want)) and np.array_equal(np.isinf(y[~gone]), np.isinf(want))
        assert (np.abs(y[~gone][fine] - want[fine]) <= np.abs(want[fine]) * 2.0 ** -23 + 1e-30).all()


def test_dropout_gradient_is_the_same_call(b):
    """The Jacobian is diagonal: differences of the (linear) forward pass along a direction against the call on that direction, and the inner
    products <dropout(x), g> and <x, dropout(g)>."""
    x, d, g = (matrix(20, 77, torch.float32, s) for s in range(3))
    h = 2.0 ** -3
    num = (f64(b.dropout(x + h * d, 0.25, draw(b))) - f64(b.dropout(x, 0.25, draw(b)))) / h
    ana = f64(b.dropout(d, 0.25, draw(b)))
    top = np.abs(f64(x)) + np.abs(f64(d))
    # x + h d is rounded once, each product once: three roundings of at most (4/3)(|x| + |d|), over h
    assert (np.abs(num - ana) <= 4 * 2.0 ** -24 * (4 / 3) * top / h + np.abs(ana) * 2.0 ** -23).all()
    left = float((b.dropout(x, 0.25, draw(b)).double() * g.double()).sum())
    right = float((x.double() * b.dropout(g, 0.25, draw(b)).double()).sum())
    assert abs(left - right) <= 2.0 ** -22 * float((x.double() * g.double()).abs().sum()) * 4 / 3


# ------------------------------------------------------------------ quantisation

def unpacked(form):
    return mo.unpack(form.codes.cpu().numpy().reshape(-1), form.scales.cpu().numpy().reshape(-1), form.rows, form.cols)


def reference(x, stochastic, p, transposed):
    """What is quantised is fp32, so the product with the dropout's scale is formed in fp32."""
    rows, cols = x.shape
    v = x.float().cpu().numpy()
    if p:
        f = int(np.rint(p * 65536))
        with np.errstate(invalid="ignore", over="ignore"):
            v = np.where(mo.numbers(*SEED, rows, cols, mo.DROPOUT) >= f, v * np.float32(65536.0 / max(1, 65536 - f)), np.float32(0))
    u = mo.numbers(*SEED, rows, cols, mo.ROUNDING) if stochastic else None
    v = v.astype(np.float64)
    return mo.encode(v.T.copy() if transposed else v, None if u is None else (u.T.copy() if transposed else u))


def check_forms(b, x, stochastic, p, view=None):
    rows, cols = x.shape
    view = x if view is None else view
    how = dict(stochastic=stochastic, p=p, draw=draw(b) if stochastic or p else None)
    a = b.mx4_quantise(view, **how)
    t = b.mx4_quantise(view, forms="cols", **how)
    a2, t2 = b.mx4_quantise(view, forms="both", **how)
    for one, two in ((a, a2), (t, t2)):
        assert one[:2] == two[:2] and torch.equal(one.codes, two.codes) and torch.equal(one.scales, two.scales)
    for form, transposed in ((a, False), (t, True)):
        assert (form.rows, form.cols) == ((cols, rows) if transposed else (rows, cols))
        codes, scales = unpacked(form)
        want_codes, want_scales = reference(x, stochastic, p, transposed)
        assert np.array_equal(scales, want_scales), np.argwhere(scales != want_scales)[:3]
        assert np.array_equal(codes, want_codes), np.argwhere(codes != want_codes)[:3]
        got = b.mx4_dequantise(form)
        assert got.shape == (form.rows, form.cols)
        with np.errstate(over="ignore"):   # (values of 2^128, to which what lies within half a step of it is rounded, are infinite in fp32)
            assert np.array_equal(got.cpu().numpy(), mo.decode(codes, scales).astype(np.float32), equal_nan=True)
    return a, t


QSHAPES = [(1, 1), (1, 31), (1, 32), (1, 33), (3, 128), (7, 1600), (129, 65), (257, 100), (128, 128), (64, 256), (200, 515), (5, 127), (500, 3), (2, 4097), (96, 96), (1030, 40), (65, 1301)]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows,cols", QSHAPES)
@pytest.mark.parametrize("stochastic,p", [(False, 0.0), (True, 0.0), (True, 0.1), (False, 0.6)])
def test_quantise(b, rows, cols, dtype, stochastic, p):
    check_forms(b, matrix(rows, cols, dtype), stochastic, p)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("front", [0, 1, 2, 4, 5, 8])
def test_quantise_strided(b, dtype, front):
    for rows, cols in ((70, 200), (33, 64), (5, 1301), (130, 31)):
        x = matrix(rows, cols, dtype)
        check_forms(b, x, True, 0.2, strided(x, front, 3)[0])
        check_forms(b, x, False, 0.0, strided(x, front, 8 - front % 8)[0])


@pytest.mark.parametrize("stochastic", [False, True])
def test_quantise_blocks_at_the_edges(b, stochastic):
    x = matrix(70, 160, torch.float32)
    x[0, :32] = 0.0
    x[1, :64] = -0.0
    x[2, 5] = float("nan")
    x[3, 40] = float("inf")
    x[4, 70] = -float("inf")
    x[5] = torch.finfo(torch.float32).max
    x[6] = torch.finfo(torch.float32).min
    x[7] = 1e-45
    x[8, ::3] = -3e-45
    x[9] *= 2.0 ** -135
    x[10, 0], x[10, 1] = 3e38, 1e-40
    x[11, :4] = torch.tensor([6.0, 6.0000005, 1.5, 0.75], device="cuda")
    x[12] = 5.0
    x[13, :32] = 0.25
    x[13, 0] = 6.0
    for row in range(14, 70):                        # ties everywhere
        x[row] = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0], device="cuda").repeat(20) * 2.0 ** (row - 40)
    a, t = check_forms(b, x, stochastic, 0.0)
    assert torch.isnan(b.mx4_dequantise(a)[2, :32]).all() and not torch.isnan(b.mx4_dequantise(a)[2, 32:]).any()
    check_forms(b, x, stochastic, 0.5)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("stochastic,p", [(False, 0.0), (True, 0.0), (False, 0.5), (True, 0.5)])
@pytest.mark.parametrize("pad", [0, 8, 1])
def test_quantise_16_bit_blocks_at_the_edges(b, dtype, stochastic, p, pad):
    tiny = {torch.bfloat16: 2.0 ** -133, torch.float16: 2.0 ** -24}[dtype]   # the least subnormal
    x = matrix(70, 192, dtype)
    x[0, :32] = 0.0
    x[1, :64] = -0.0
    x[2, 5] = float("nan")
    x[3, 40] = float("inf")
    x[4, 71] = -float("inf")
    x[5] = torch.finfo(dtype).max
    x[6] = torch.finfo(dtype).min
    x[7] = tiny
    x[8, ::3] = -3 * tiny
    x[9] = (matrix(1, 192, torch.float32)[0] * 2.0 ** -110).to(dtype)
    x[10, 0], x[10, 1] = torch.finfo(dtype).max, tiny
    x[12] = 5.0
    x[13, :32] = 0.25
    x[13, 0] = 6.0
    for row in range(14, 44):                        # ties everywhere
        x[row] = (torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0], device="cuda").repeat(24) * 2.0 ** (row - 30)).to(dtype)
    x[64:] *= 64 * tiny                              # columns whose last rows are subnormals
    check_forms(b, x, stochastic, p, strided(x, 0, pad)[0] if pad else None)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_dequantise_to_shorter_types(b, dtype):
    x = matrix(37, 205, torch.float32)
    a = b.mx4_quantise(x)
    assert torch.equal(b.mx4_dequantise(a, dtype=dtype), b.mx4_dequantise(a).to(dtype))


def test_forms_of_nothing(b):
    for shape in ((0, 40), (40, 0), (0, 0)):
        a, t = b.mx4_quantise(torch.empty(shape, device="cuda"), forms="both")
        assert (a.rows, a.cols) == shape and (t.cols, t.rows) == shape
        assert b.mx4_dequantise(a).shape == shape
        assert b.mx4_matmul(a, a, dtype=torch.float32).shape == (shape[0], shape[0])
        assert not b.mx4_matmul(a, a, dtype=torch.float32).any()


def test_quantise_refusals(b):
    x = matrix(8, 64, torch.float32)
    for call in (lambda: b.mx4_quantise(x, forms="row"), lambda: b.mx4_quantise(x, stochastic=True), lambda: b.mx4_quantise(x, p=0.5),
                 lambda: b.mx4_quantise(x.t()), lambda: b.mx4_quantise(x, p=1.5, draw=draw(b)), lambda: b.mx4_quantise(x.double()),
                 lambda: b.mx4_dequantise(b.mx4_quantise(x), dtype=torch.float64),
                 lambda: b.mx4_dequantise(b.mx4_quantise(x)._replace(rows=9)), lambda: b.mx4_matmul(b.mx4_quantise(x), b.mx4_quantise(x[:, :60])),
                 lambda: b.mx4_matmul(b.mx4_quantise(x), b.mx4_quantise(x)._replace(scales=torch.zeros(511, dtype=torch.uint8, device="cuda")))):
        with pytest.raises(b.ConEFError) as e:
            call()
        assert e.value.code == b.ERR_INVALID_ARG
    odd = torch.zeros(8 * 32 + 1, dtype=torch.uint8, device="cuda")[1:]
    with pytest.raises(b.ConEFError):
        b.mx4_dequantise(b.mx4_quantise(x)._replace(codes=odd))


# ------------------------------------------------------------------ products

def check_product(b, a, c, dtype):
    """Products of codes and scales are exact; each of the k sums in fp32 is off by 2^-23 of the sum of sizes at most (2^-24 where it
    rounds, twice that where it drops bits), and the result is rounded to the type once."""
    got = f64(b.mx4_matmul(a, c, dtype=dtype))
    va, vc = mo.decode(*unpacked(a)), mo.decode(*unpacked(c))
    want, size = va @ vc.T, np.abs(va) @ np.abs(vc).T
    tol = a.cols * 2.0 ** -23 * size + np.abs(want) * EPS[dtype] * 1.001 + TINY[dtype]
    assert got.shape == want.shape
    off = ~(np.abs(got - want) <= tol)
    assert not off.any(), (np.argwhere(off)[:3], got[off][:3], want[off][:3])


PSHAPES = [(1, 64, 32), (1, 6400, 1600), (1, 1, 1), (2, 100, 33), (7, 129, 257), (16, 64, 1600), (17, 65, 64), (33, 300, 95), (64, 64, 128), (65, 640, 651), (127, 1111, 31),
           (128, 128, 256), (129, 257, 1024), (300, 200, 512), (256, 512, 1600), (1111, 261, 651), (1000, 130, 4100), (5, 70, 20000)]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("m,n,k", PSHAPES)
def test_product(b, m, n, k, dtype):
    a = b.mx4_quantise(matrix(m, k, torch.float32))
    c = b.mx4_quantise(matrix(n, k, torch.float32, 1, 0.02))
    check_product(b, a, c, dtype)


@pytest.mark.parametrize("m,n,k", [(3, 100, 96), (150, 140, 320)])
def test_product_of_small_integers_is_exact(b, m, n, k):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(1)
    a, c = (torch.randint(-4, 5, (r, k), generator=gen, device="cuda").float() for r in (m, n))
    a[:, ::32], c[:, ::32] = 4.0, -4.0          # every block has scale 1 (4 <= 6, 4 > 3)
    got = b.mx4_matmul(b.mx4_quantise(a), b.mx4_quantise(c), dtype=torch.float32)
    assert torch.equal(got.double(), a.double() @ c.double().t())


@pytest.mark.parametrize("m,n", [(4, 200), (140, 200)])
def test_product_of_values_that_are_not_finite(b, m, n):
    a, c = matrix(m, 200, torch.float32), matrix(n, 200, torch.float32, 1)
    a[2, 77], c[5, 3], a[3] = float("nan"), float("inf"), 0.0
    got = b.mx4_matmul(b.mx4_quantise(a), b.mx4_quantise(c), dtype=torch.float32)
    bad = torch.zeros(m, n, dtype=torch.bool, device="cuda")
    bad[2], bad[:, 5] = True, True
    assert torch.equal(torch.isnan(got), bad)
    a[2, 77], c[5, 3] = 1.0, 1.0
    big = b.mx4_matmul(b.mx4_quantise(a.abs() * 1e30), b.mx4_quantise(c.abs() * 1e30), dtype=torch.float32)
    assert torch.isinf(big[0]).all() and not big[3].any()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("tokens,inner,outer", [(200, 160, 320), (8, 1600, 200)])
def test_a_linear_layer_forward_and_backward(b, tokens, inner, outer, dtype):
    """Dropout, both forms of activations, weights and gradients, and the three products of a training step."""
    x, w, dy = matrix(tokens, inner, dtype), matrix(outer, inner, dtype, 1, 0.02), matrix(tokens, outer, dtype, 2, 1e-3)
    xr, xt = b.mx4_quantise(x, forms="both", stochastic=True, p=0.1, draw=draw(b))
    wr, wt = b.mx4_quantise(w, forms="both")
    gr, gt = b.mx4_quantise(dy, forms="both", stochastic=True, draw=b.Draw(77, 1, 6, 9))
    check_product(b, xr, wr, dtype)          # y = x w^T
    check_product(b, gr, wt, dtype)          # dx = dy w
    check_product(b, gt, xt, dtype)          # dw = dy^T x
    dx = b.dropout(b.mx4_matmul(gr, wt, dtype=dtype), 0.1, draw(b))
    assert not dx[torch.from_numpy(mo.numbers(*SEED, tokens, inner, mo.DROPOUT) < round(6553.6)).cuda()].any()


def test_on_another_stream_and_in_a_graph(b):
    x = matrix(300, 700, torch.bfloat16)
    w = b.mx4_quantise(matrix(129, 700, torch.bfloat16, 1))

    def chain(stream=None):
        y = b.dropout(x, 0.1, draw(b), add=x, stream=stream)
        r, t = b.mx4_quantise(y, forms="both", stochastic=True, p=0.2, draw=draw(b), stream=stream)
        return [y, r.codes, r.scales, t.codes, t.scales, b.mx4_dequantise(t, stream=stream), b.mx4_matmul(r, w, stream=stream)]

    want = chain()
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    got = chain(s)
    s.synchronize()
    assert all(torch.equal(p, q) for p, q in zip(want, got))
    with torch.cuda.stream(s):
        got = chain()
    s.synchronize()
    assert all(torch.equal(p, q) for p, q in zip(want, got))
    keep = x.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = chain()
    x.copy_(matrix(300, 700, torch.bfloat16, 9))
    graph.replay()
    again = [t.clone() for t in out]
    fresh = chain()
    assert all(torch.equal(p, q) for p, q in zip(fresh, again))
    x.copy_(keep)
    graph.replay()
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(p, q) for p, q in zip(want, out))


def test_behind_a_kernel_that_writes_the_input_late(b):
    """The launches may come onto the SMs before the kernel ahead has ended; what they read has to be its result."""
    src = matrix(64, 512, torch.float32)
    a = torch.randn(4096, 4096, device="cuda")
    want = [b.dropout(src, 0.5, draw(b)), b.mx4_dequantise(b.mx4_quantise(src)), b.mx4_matmul(b.mx4_quantise(src), b.mx4_quantise(src))]
    for _ in range(3):
        x = torch.zeros_like(src)
        torch.cuda.synchronize()
        for _ in range(4):
            a = a @ a * 1e-4
        x.copy_(src)
        got = [b.dropout(x, 0.5, draw(b)), b.mx4_dequantise(b.mx4_quantise(x)), b.mx4_matmul(b.mx4_quantise(x), b.mx4_quantise(x))]
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(want, got))


def test_two_chains_at_once(b):
    """Calls on two streams without an order between them: none keeps anything that the other could find."""
    streams = [torch.cuda.Stream() for _ in range(2)]
    jobs = []
    for i, (m, n, k) in enumerate([(1000, 700, 1600), (300, 64, 320)]):
        jobs.append((matrix(m, k, torch.bfloat16, i), b.mx4_quantise(matrix(n, k, torch.bfloat16, 7 + i)), b.Draw(1, 0, i, 0)))

    def chain(x, w, d, stream=None):
        y = b.dropout(x, 0.1, d, stream=stream)
        r, t = b.mx4_quantise(y, forms="both", stochastic=True, p=0.2, draw=d, stream=stream)
        return b.mx4_matmul(r, w, dtype=torch.float32, stream=stream), b.mx4_dequantise(t, stream=stream)

    want = [chain(*j) for j in jobs]
    torch.cuda.synchronize()
    got = [[chain(*j, stream=s) for _ in range(20)] for j, s in zip(jobs, streams)]
    both = []
    for _ in range(20):
        for j, s in zip(jobs, streams):
            both.append((j, chain(*j, stream=s)))
    torch.cuda.synchronize()
    for w, runs in zip(want, got):
        for r in runs:
            assert all(torch.equal(p, q) for p, q in zip(w, r))
    for i, (_, r) in enumerate(both):
        assert all(torch.equal(p, q) for p, q in zip(want[i % 2], r))


def test_a_tensor_given_up_while_another_stream_works_on_it(b):
    s = torch.cuda.Stream()
    a = torch.randn(4096, 4096, device="cuda")
    x = matrix(512, 1600, torch.float32)
    want = b.dropout(x, 0.5, draw(b))
    torch.cuda.synchronize()
    for _ in range(4):
        y = x.clone()
        torch.cuda.synchronize()
        with torch.cuda.stream(s):
            for _ in range(3):
                a = a @ a * 1e-4
        got = b.dropout(y, 0.5, draw(b), stream=s)
        del y
        z = torch.full((512, 1600), 9.0, device="cuda")       # would take y's memory
        torch.cuda.synchronize()
        assert torch.equal(got, want)
        del z


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("extra,front", [(0, 0), (1, 0), (3, 1), (8, 0), (16, 8), (13, 5)])
@pytest.mark.parametrize("m,n,k", [(5, 70, 64), (140, 131, 96), (300, 256, 300)])
def test_results_with_rows_further_apart(b, dtype, extra, front, m, n, k):
    """Products and values into the columns of a wider matrix, through the C interface: what lies between the rows stays."""
    a, c = b.mx4_quantise(matrix(m, k, torch.float32)), b.mx4_quantise(matrix(n, k, torch.float32, 1))
    ld, code = n + front + extra, {torch.float32: b.F32, torch.bfloat16: b.BF16, torch.float16: b.F16}[dtype]
    wide = torch.full((m + 2, ld), 7.0, dtype=dtype, device="cuda")
    at = wide.data_ptr() + (ld + front) * wide.element_size()
    assert b.lib.conef_mx4_matmul(a.codes.data_ptr(), a.scales.data_ptr(), m, c.codes.data_ptr(), c.scales.data_ptr(), n, k, at, code, ld, b._stream_handle(None)) == b.OK
    inner = wide[1:-1, front:front + n]
    assert torch.equal(inner, b.mx4_matmul(a, c, dtype=dtype))
    inner.fill_(7.0)
    assert (wide == 7).all()
    q = b.mx4_quantise(matrix(m, n, torch.float32, 2))
    assert b.lib.conef_mx4_dequantise(q.codes.data_ptr(), q.scales.data_ptr(), m, n, at, code, ld, b._stream_handle(None)) == b.OK
    assert torch.equal(inner, b.mx4_dequantise(q, dtype=dtype))
    inner.fill_(7.0)
    assert (wide == 7).all()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows,cols", [(5000, 1), (3000, 2), (1, 70000), (2, 33333), (129, 8192)])
def test_narrow_and_long_matrices(b, dtype, rows, cols):
    x = matrix(rows, cols, dtype)
    check_dropout(b.dropout(x, 0.3, draw(b)), x, 0.3)
    codes, scales = unpacked(b.mx4_quantise(x, stochastic=True, p=0.3, draw=draw(b)))
    want = reference(x, True, 0.3, False)
    assert np.array_equal(codes, want[0]) and np.array_equal(scales, want[1])
    a, t = b.mx4_quantise(x, forms="both")
    for form, transposed in ((a, False), (t, True)):
        got, want = unpacked(form), reference(x, False, 0.0, transposed)
        assert np.array_equal(got[0], want[0]) and np.array_equal(got[1], want[1])
        assert np.array_equal(f64(b.mx4_dequantise(form)), mo.decode(*want))


def test_a_row_of_a_larger_tensor_and_an_array_off_a_boundary(b):
    whole = matrix(1, 40 * 999 + 5, torch.bfloat16)[0]
    x = whole[5:].view(40, 999)
    how = dict(stochastic=True, p=0.25, draw=draw(b))
    for form, other in zip(b.mx4_quantise(x, forms="both", **how), b.mx4_quantise(x.clone(), forms="both", **how)):
        assert torch.equal(form.codes, other.codes) and torch.equal(form.scales, other.scales)

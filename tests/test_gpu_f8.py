"""Quantisation to 8-bit floats with block scales and products of what it leaves, against the plain statement in 64 bits."""
import numpy as np
import pytest
import torch

from oracle import f8_oracle as fo

pytestmark = pytest.mark.gpu

EPS = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}   # half a step, relative
TINY = {torch.float32: 2.0 ** -149, torch.bfloat16: 2.0 ** -133, torch.float16: 2.0 ** -24}
DTYPES = [torch.float32, torch.bfloat16, torch.float16]
KINDS = ["e4m3", "e5m2"]


@pytest.fixture(scope="module")
def b():
    from paper_2312_08538_b200 import binding
    return binding


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


def check_form(form, x, kind, square=False):
    """Codes and scales are those of x (float64), bit for bit."""
    assert (form.rows, form.cols, form.kind) == (*x.shape, kind)
    codes, scales = fo.unpack(form.codes.cpu().numpy(), form.scales.cpu().numpy(), *x.shape)
    want, want_scales = fo.encode(x, kind, square)
    assert np.array_equal(scales, want_scales), np.argwhere(scales != want_scales)[:3]
    assert np.array_equal(codes, want), (np.argwhere(codes != want)[:3], codes[codes != want][:3], want[codes != want][:3])


def check_forms(b, given, x, kind, square=False):
    x = f64(x)
    check_form(b.f8_quantise(given, kind=kind, square=square), x, kind, square)
    check_form(b.f8_quantise(given, "cols", kind, square), x.T.copy(), kind, square)
    r, t = b.f8_quantise(given, "both", kind, square)
    check_form(r, x, kind, square)
    check_form(t, x.T.copy(), kind, square)


SHAPES = [(1, 1), (1, 3), (7, 1600), (5, 33), (128, 128), (129, 127), (33, 1301), (300, 8), (1000, 2), (1, 4100), (130, 4097), (257, 512), (513, 640)]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows,cols", SHAPES)
def test_forms(b, rows, cols, dtype):
    x = matrix(rows, cols, dtype)
    for kind in KINDS:
        check_forms(b, x, x, kind)
        check_forms(b, x, x, kind, True)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("front,behind", [(0, 8), (8, 8), (16, 16), (1, 2), (3, 5), (4, 4)])
def test_forms_of_strided_rows(b, dtype, front, behind):
    for rows, cols in ((37, 300), (130, 528)):
        x = matrix(rows, cols, dtype)
        view, wide = strided(x, front, behind)
        check_forms(b, view, x, "e4m3")
        check_forms(b, view, x, "e5m2", True)
        assert (wide[:, :front] == 7).all() and (wide[:, front + cols:] == 7).all()


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("dtype", DTYPES)
def test_borders(b, dtype, kind):
    """Ties, the largest value and what lies next to it, subnormals, zeros of both signs, the ends of the range."""
    g = fo.grid(kind)
    lines = []
    for power in (0, -5, 3, -140, -126, -110, 100, 119):
        v = np.concatenate([g, (g[:-1] + g[1:]) / 2, np.nextafter(g[-1], [0, 1e9]), [0.0]])
        v = np.concatenate([v, -v])
        for q in range(0, v.size, 127):
            part = np.zeros(128)
            part[:v[q:q + 127].size] = v[q:q + 127]
            part[127] = g[-1] if q % 2 == 0 else g[-1] * (1 + 2.0 ** -7)
            with np.errstate(over="ignore"):
                lines.append(np.ldexp(part, power))
    x = torch.from_numpy(np.array(lines)).float().cuda()
    x = torch.where(torch.isfinite(x), x, 0.0).to(dtype)
    x = torch.where(torch.isfinite(x), x, torch.zeros_like(x))
    check_forms(b, x, x, kind)
    wide = torch.cat([x, x.flip(0)], 1)[:, 1:]   # (elements one by one)
    check_forms(b, wide, wide, kind)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("dtype", DTYPES)
def test_blocks_with_infinities_and_nan(b, dtype, kind):
    for cols in (640, 641):
        x = matrix(140, cols, dtype)
        x[3, 5], x[77, 300], x[139, cols - 1], x[0, 128] = float("inf"), float("nan"), float("-inf"), float("nan")
        check_forms(b, x, x, kind)
        check_forms(b, x, x, kind, True)
        v = b.f8_dequantise(b.f8_quantise(x, kind=kind))
        assert torch.isnan(v[3, :128]).all() and torch.isnan(v[77, 256:384]).all() and int(torch.isnan(v).any(1).sum()) == 4


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("rows,cols", [(1, 1), (7, 1600), (33, 1301), (200, 640), (130, 515)])
def test_values(b, rows, cols, kind, dtype):
    x = matrix(rows, cols, torch.float32, scale=0.01)
    form = b.f8_quantise(x, kind=kind)
    want = fo.decode(*fo.encode(f64(x), kind), kind)
    got = f64(b.f8_dequantise(form, dtype))
    if dtype == torch.float16:   # rounded once
        assert (np.abs(got - want) <= np.abs(want) * EPS[dtype] + TINY[dtype] / 2).all()
    else:
        assert np.array_equal(got, want)


def test_no_rows_or_columns(b):
    for rows, cols in ((0, 5), (5, 0), (0, 0)):
        x = torch.empty(rows, cols, device="cuda")
        r, t = b.f8_quantise(x, "both")
        assert b.f8_dequantise(r).shape == (rows, cols) and b.f8_dequantise(t).shape == (cols, rows)
    assert not b.f8_matmul(b.f8_quantise(torch.empty(3, 0, device="cuda")), b.f8_quantise(torch.empty(130, 0, device="cuda"))).any()
    assert b.f8_matmul(b.f8_quantise(torch.empty(0, 7, device="cuda")), b.f8_quantise(torch.ones(4, 7, device="cuda"))).shape == (0, 4)


# ------------------------------------------------------------------ products

def check_product(got, a, c, dtype):
    """a, c: the values (float64).  Sums of exact products in fp32: a rounding of each 32 products' sum and of the running one, by a step of 2^-23 at most
    where the hardware cuts off, relative to what the sums have grown to; then one rounding to the type."""
    want, size = a @ c.T, np.abs(a) @ np.abs(c).T
    tol = np.abs(want) * EPS[dtype] * 1.001 + size * 2.0 ** -23 * (a.shape[1] / 32 + 2) + TINY[dtype]
    got = f64(got)
    off = ~(np.abs(got - want) <= tol)
    assert got.shape == want.shape and not off.any(), (np.argwhere(off)[:3], got[off][:3], want[off][:3])


def values(form):
    return fo.decode(*fo.unpack(form.codes.cpu().numpy(), form.scales.cpu().numpy(), form.rows, form.cols), form.kind)


PRODUCTS = [(1, 1, 1), (1, 64, 32), (2, 3, 500), (128, 64, 128), (129, 65, 129), (1, 640, 160), (70, 200, 33), (300, 300, 160), (257, 513, 1600), (111, 260, 651), (16, 1000, 4100)]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("m,n,k", PRODUCTS)
def test_product(b, m, n, k, dtype):
    for kinds in (("e4m3", "e4m3"), ("e5m2", "e4m3"), ("e4m3", "e5m2"), ("e5m2", "e5m2")):
        a, c = b.f8_quantise(matrix(m, k, torch.float32), kind=kinds[0]), b.f8_quantise(matrix(n, k, torch.float32, 1, 0.02), kind=kinds[1])
        check_product(b.f8_matmul(a, c, dtype), values(a), values(c), dtype)


@pytest.mark.parametrize("m,n,k", [(3330, 4113, 260), (8192, 640, 300), (2048, 2048, 1600), (40001, 187, 130), (1000, 1600, 1600)])
def test_product_of_every_kind_of_tile(b, m, n, k):
    a, c = b.f8_quantise(matrix(m, k, torch.bfloat16), kind="e5m2"), b.f8_quantise(matrix(n, k, torch.bfloat16, 1, 0.02))
    check_product(b.f8_matmul(a, c, torch.bfloat16), values(a), values(c), torch.bfloat16)
    check_product(b.f8_matmul(a, c, torch.float32), values(a), values(c), torch.float32)


def test_product_scales_and_single_elements(b):
    """Each element against each: a one at (r, c) of A and B in turn, under scales from 2^-100 to 2^100."""
    k = 1100
    a, c = torch.zeros(k, k, device="cuda"), torch.zeros(k, k, device="cuda")
    e = (torch.arange(k, device="cuda") * 37 % 101 - 50).float()
    a[torch.arange(k), torch.arange(k)] = torch.exp2(e)
    c[torch.arange(k), (torch.arange(k) * 7 + 3) % k] = torch.exp2(-e * 0.5)
    fa, fc = b.f8_quantise(a), b.f8_quantise(c, kind="e5m2")
    assert np.array_equal(values(fa), f64(a))
    check_product(b.f8_matmul(fa, fc, torch.float32), values(fa), values(fc), torch.float32)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("m", [1, 2, 7, 8, 9, 15, 16, 17])
def test_product_of_few_rows(b, m, dtype):
    """... of either side."""
    for n, k in ((1, 1), (17, 33), (100, 1300), (640, 128), (301, 4100)):
        a, c = b.f8_quantise(matrix(m, k, torch.float32), kind="e5m2"), b.f8_quantise(matrix(n, k, torch.float32, 1, 0.02))
        got = b.f8_matmul(a, c, dtype)
        check_product(got, values(a), values(c), dtype)
        turned = b.f8_matmul(c, a, dtype)
        check_product(turned, values(c), values(a), dtype)


def test_product_of_few_rows_with_nan_blocks_and_far_scales(b):
    for m in (3, 12):
        x, w = matrix(m, 640, torch.bfloat16), matrix(70, 640, torch.bfloat16, 1)
        x[1, 200] = float("nan")
        w[66, 639] = float("inf")
        out = b.f8_matmul(b.f8_quantise(x), b.f8_quantise(w))
        bad = torch.zeros_like(out, dtype=torch.bool)
        bad[1], bad[:, 66] = True, True
        assert torch.equal(torch.isnan(out), bad)
        for up, down in ((2.0 ** 118, 2.0 ** -118), (2.0 ** -120, 2.0 ** 119), (2.0 ** 60, 2.0 ** -100)):
            a, c = b.f8_quantise(matrix(m, 300, torch.float32).clamp(-200, 200) * up), b.f8_quantise(matrix(40, 300, torch.float32, 1).clamp(-200, 200) * down)
            check_product(b.f8_matmul(a, c, torch.float32), values(a), values(c), torch.float32)


def test_product_with_nan_blocks(b):
    x, w = matrix(140, 640, torch.bfloat16), matrix(70, 640, torch.bfloat16, 1)
    x[5, 200] = float("nan")
    w[66, 639] = float("inf")
    out = b.f8_matmul(b.f8_quantise(x), b.f8_quantise(w))
    bad = torch.zeros_like(out, dtype=torch.bool)
    bad[5], bad[:, 66] = True, True
    assert torch.equal(torch.isnan(out), bad)


def test_a_layer_and_its_gradients(b):
    """Y = X W^T, dX = dY W, dW = dY^T X from the forms that one reading of each leaves."""
    x, w, dy = matrix(300, 200, torch.bfloat16), matrix(150, 200, torch.bfloat16, 1), matrix(300, 150, torch.bfloat16, 2)
    (xr, xt), (wr, wt), (gr, gt) = b.f8_quantise(x, "both"), b.f8_quantise(w, "both", square=True), b.f8_quantise(dy, "both", kind="e5m2")
    assert np.array_equal(values(wr), values(wt).T)
    for got, p, q in ((b.f8_matmul(xr, wr), xr, wr), (b.f8_matmul(gr, wt), gr, wt), (b.f8_matmul(gt, xt), gt, xt)):
        check_product(got, values(p), values(q), torch.bfloat16)
    # ... and near the products of what was quantised: a rounding of either factor, half a step of 2^-3 (e4m3) or 2^-2 (e5m2) relative
    near = f64(x) @ f64(w).T
    assert np.linalg.norm(f64(b.f8_matmul(xr, wr)) - near) <= (2 * 2.0 ** -4 + 2.0 ** -7) * np.linalg.norm(np.abs(f64(x)) @ np.abs(f64(w)).T)


# ------------------------------------------------------------------ streams, graphs, refusals

def test_on_another_stream(b):
    x, w = matrix(300, 650, torch.bfloat16), matrix(200, 650, torch.bfloat16, 1)
    want = b.f8_matmul(b.f8_quantise(x), b.f8_quantise(w))
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    got = b.f8_matmul(b.f8_quantise(x, stream=s), b.f8_quantise(w, stream=s), stream=s)
    shown = b.f8_dequantise(b.f8_quantise(x, stream=s), stream=s)
    s.synchronize()
    assert torch.equal(got, want) and torch.equal(shown, b.f8_dequantise(b.f8_quantise(x)))


def test_in_a_graph(b):
    x, w = matrix(300, 650, torch.bfloat16), matrix(200, 650, torch.bfloat16, 1)

    def run():
        (a, t), c = b.f8_quantise(x, "both"), b.f8_quantise(w, square=True)
        return b.f8_matmul(a, c), b.f8_dequantise(t)

    run()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        outs = run()
    for seed in range(3):
        x.copy_(matrix(300, 650, torch.bfloat16, seed + 5))
        g.replay()
        assert all(torch.equal(o, want) for o, want in zip(outs, run()))


def test_refusals(b):
    x = matrix(40, 64, torch.float32)
    form = b.f8_quantise(x)
    bad = [lambda: b.f8_quantise(x, "sideways"), lambda: b.f8_quantise(x, kind="e3m4"), lambda: b.f8_quantise(x.t()), lambda: b.f8_quantise(x.long()),
           lambda: b.f8_quantise(x.clone().requires_grad_()), lambda: b.f8_dequantise(form, torch.float64), lambda: b.f8_dequantise(form._replace(kind="e2m5")),
           lambda: b.f8_dequantise(form._replace(rows=41)), lambda: b.f8_matmul(form, b.f8_quantise(x[:, :60])), lambda: b.f8_matmul(form, form, torch.int32),
           lambda: b.f8_matmul(form, form._replace(scales=form.scales[:-1]))]
    for call in bad:
        with pytest.raises(b.ConEFError) as e:
            call()
        assert e.value.code == b.ERR_INVALID_ARG


def test_nothing_runs_out(b):
    before = b.f8_timeouts()
    a, c = b.f8_quantise(matrix(3330, 2100, torch.bfloat16)), b.f8_quantise(matrix(4113, 2100, torch.bfloat16, 1))
    assert not torch.isnan(b.f8_matmul(a, c)).any()
    assert b.f8_timeouts() == before


@pytest.mark.parametrize("m,n,k", [(24, 200, 6400), (33, 129, 6400), (64, 100, 4100), (65, 100, 4100), (64, 64, 20000), (19, 777, 1300), (9, 60, 33)])
def test_product_of_some_rows(b, m, n, k):
    """... by groups of eight against a long k, and either side's."""
    for kinds in (("e4m3", "e5m2"), ("e5m2", "e4m3")):
        a, c = b.f8_quantise(matrix(m, k, torch.float32), kind=kinds[0]), b.f8_quantise(matrix(n, k, torch.float32, 1, 0.02), kind=kinds[1])
        for got, x, y in ((b.f8_matmul(a, c, torch.float32), a, c), (b.f8_matmul(c, a, torch.float32), c, a)):
            check_product(got, values(x), values(y), torch.float32)


def test_product_of_some_rows_into_a_wider_matrix(b):
    a, c = b.f8_quantise(matrix(27, 2000, torch.bfloat16)), b.f8_quantise(matrix(90, 2000, torch.bfloat16, 1))
    for p, q in ((a, c), (c, a)):
        wide = torch.full((p.rows + 2, q.rows + 3), 7.0, device="cuda")
        assert b.lib.conef_f8_matmul(p.codes.data_ptr(), p.scales.data_ptr(), b.E4M3, p.rows, q.codes.data_ptr(), q.scales.data_ptr(), b.E4M3, q.rows, 2000, wide[1:, 1:].data_ptr(),
                                     b.F32, wide.shape[1], b._stream_handle(None)) == b.OK
        assert torch.equal(wide[1:-1, 1:-2], b.f8_matmul(p, q, torch.float32))
        wide[1:-1, 1:-2] = 7.0
        assert (wide == 7.0).all()


def test_product_of_some_rows_with_a_nan_block(b):
    x, w = matrix(30, 3000, torch.bfloat16), matrix(70, 3000, torch.bfloat16, 1)
    x[29, 2999], w[66, 639] = float("nan"), float("inf")
    for out, i, j in ((b.f8_matmul(b.f8_quantise(x), b.f8_quantise(w)), 29, 66), (b.f8_matmul(b.f8_quantise(w), b.f8_quantise(x)), 66, 29)):
        bad = torch.zeros_like(out, dtype=torch.bool)
        bad[i], bad[:, j] = True, True
        assert torch.equal(torch.isnan(out), bad)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("m,n,k", [(100, 1600, 6400), (130, 77, 8192), (200, 130, 20000), (256, 256, 33001), (65, 65, 4097), (129, 513, 2048), (300, 700, 5000), (768, 768, 8192)])
def test_product_of_few_tiles_against_a_long_k(b, m, n, k, dtype):
    """... where thread blocks share a tile along k."""
    a, c = b.f8_quantise(matrix(m, k, torch.bfloat16), kind="e5m2"), b.f8_quantise(matrix(n, k, torch.bfloat16, 1, 0.02))
    got = b.f8_matmul(a, c, dtype)
    check_product(got, values(a), values(c), dtype)
    assert all(torch.equal(b.f8_matmul(a, c, dtype), got) for _ in range(3))


def test_product_of_few_tiles_into_a_wider_matrix_with_a_nan_block(b):
    x, w = matrix(140, 9000, torch.bfloat16), matrix(90, 9000, torch.bfloat16, 1)
    x[139, 8999], w[66, 639] = float("nan"), float("inf")
    p, q = b.f8_quantise(x), b.f8_quantise(w)
    wide = torch.full((142, 93), 7.0, device="cuda")
    assert b.lib.conef_f8_matmul(p.codes.data_ptr(), p.scales.data_ptr(), b.E4M3, 140, q.codes.data_ptr(), q.scales.data_ptr(), b.E4M3, 90, 9000, wide[1:, 1:].data_ptr(), b.F32, 93,
                                 b._stream_handle(None)) == b.OK
    bad = torch.zeros(140, 90, dtype=torch.bool, device="cuda")
    bad[139], bad[:, 66] = True, True
    assert torch.equal(torch.isnan(wide[1:-1, 1:-2]), bad)
    wide[1:-1, 1:-2] = 7.0
    assert (wide == 7.0).all()

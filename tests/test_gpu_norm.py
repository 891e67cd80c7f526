"""Root-mean-square norms with the residual's addition, their 8-bit forms and their gradient, against the plain statement in 64 bits."""
import ctypes as C

import numpy as np
import pytest
import torch

from oracle import f8_oracle as fo
from tests.test_gpu_f8 import DTYPES, EPS, TINY, b, check_form, f64, matrix, strided  # noqa: F401  (b: a fixture)

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
SHAPES = [(1, 1), (1, 1600), (3, 5), (7, 512), (5, 513), (300, 64), (301, 1301), (300, 2048), (2, 2049), (9, 4100), (6, 8192), (3, 8193), (2, 20001), (700, 768), (5, 20480)]


def weight(cols, dtype, seed=0):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(cols + seed)
    return (1.0 + 0.3 * torch.randn(cols, generator=gen, device="cuda")).to(dtype)


def summed(x, add):
    """h as the operator rounds it."""
    return x if add is None else (x.float() + add.float()).to(x.dtype)


def check_norm(out, x, w, eps, add, forms, kind="e4m3"):
    h = summed(x, add)
    assert torch.equal(out.h, h) and out.rstd.shape == x.shape[:-1]
    want, root = fo.rms_norm(f64(h), f64(w), eps)
    exact = 1.0 / np.sqrt((f64(h) ** 2).mean(1) + eps)
    got = f64(out.rstd)
    assert (np.abs(got - exact) <= exact * U * 1.0001 + 2.0 ** -150).all()   # (64 bits, rounded once)
    stored = out.rstd.cpu().numpy()
    want = f64(h) * stored.astype(np.float64)[:, None] * f64(w)
    if forms is None:   # two roundings in fp32, one to the type
        tol = np.abs(want) * (EPS[x.dtype] + 2 * U) * 1.001 + TINY[x.dtype]
        assert (np.abs(f64(out.y) - want) <= tol).all()
        return
    both = out.y if forms == "both" else (out.y, out.y)
    if forms != "cols":
        check_form(both[0], want, kind)
    if forms != "rows":
        check_form(both[1], want.T.copy(), kind)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows,cols", SHAPES)
def test_norm(b, rows, cols, dtype):
    x, r = matrix(rows, cols, dtype), matrix(rows, cols, dtype, 1)
    for wt in {dtype, torch.float32}:
        w = weight(cols, wt)
        check_norm(b.rms_norm(x, w, 1e-5), x, w, 1e-5, None, None)
        check_norm(b.rms_norm(x, w, 1e-5, add=r), x, w, 1e-5, r, None)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows,cols", SHAPES)
def test_norm_to_8_bits(b, rows, cols, dtype):
    x, r = matrix(rows, cols, dtype), matrix(rows, cols, dtype, 1)
    for wt, forms, kind, add in ((dtype, "rows", "e4m3", r), (torch.float32, "rows", "e5m2", None), (torch.float32, "both", "e4m3", r), (dtype, "cols", "e5m2", None)):
        w = weight(cols, wt)
        check_norm(b.rms_norm(x, w, 1e-5, add=add, forms=forms, kind=kind), x, w, 1e-5, add, forms, kind)


@pytest.mark.parametrize("dtype", DTYPES)
def test_values_next_to_borders(b, dtype):
    """Rows whose root is a power of two and whose elements, times the weight, are ties of the 8-bit types: their codes are the even ones; with a weight an
    ulp off they go to their side."""
    for cols in (256, 257):
        x = torch.full((40, cols), 1.0, device="cuda")
        x[1::2] = 4.0
        g = torch.from_numpy(fo.grid("e4m3")).float().cuda()
        ties = (g[1:-1] + g[2:]) / 2
        for bump in (0.0, 2.0 ** -23, -2.0 ** -24):
            w = ties.repeat(3)[:cols] * (1.0 + bump)
            w[0] = 448.0 / 1.0
            for forms in ("rows", "both"):
                check_norm(b.rms_norm(x.to(dtype), w, 0.0, forms=forms), x.to(dtype), w, 0.0, None, forms)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("front,behind", [(0, 16), (8, 8), (1, 2), (4, 4)])
def test_strided_rows(b, dtype, front, behind):
    for rows, cols in ((37, 300), (130, 1056)):
        x, r, dy, dh = (matrix(rows, cols, dtype, i) for i in range(4))
        w = weight(cols, torch.float32)
        (xs, wide), (rs, _), (ds, _), (hs, _) = (strided(t, front, behind) for t in (x, r, dy, dh))
        out = b.rms_norm(xs, w, 1e-5, add=rs)
        check_norm(out, x, w, 1e-5, r, None)
        check_norm(b.rms_norm(x, w, 1e-5, add=rs, forms="both"), x, w, 1e-5, r, "both")
        check_grad(b.rms_norm_grad(ds, out.h, w, out.rstd, add=hs), dy, out.h, w, out.rstd, dh)
        check_grad(b.rms_norm_grad(dy, xs, w, out.rstd), dy, x, w, out.rstd, None)
        assert (wide[:, :front] == 7).all() and (wide[:, front + cols:] == 7).all()


def check_grad(got, dy, h, w, rstd, add):
    dx, dw = got
    d, v, ww, r = f64(dy), f64(h), f64(w), rstd.cpu().numpy()
    want, want_w = fo.rms_norm_grad(d, v, ww, r)
    n, g = v * r.astype(np.float64)[:, None], d * ww
    size = np.abs(g * n).mean(1, keepdims=True)
    # fp32: n, g, the products and their differences a rounding each; the mean 16 + 5 + 16 additions deep (or, of rows beyond 8192 columns, an addition more per
    # 4096 of them), and its division; then the sum with what else reached h
    deep = 42 + h.shape[1] / 4096
    tol = r.astype(np.float64)[:, None] * (np.abs(g) * 3 + np.abs(n) * size * deep + np.abs(n) * np.abs((g * n).mean(1, keepdims=True)) * 5) * U
    if add is not None:
        want = want + f64(add)
        tol = tol + (np.abs(want) + np.abs(f64(add))) * U
    tol = tol * 1.01 + np.abs(want) * (EPS[dy.dtype] + U) * 1.001 + TINY[dy.dtype]
    off = ~(np.abs(f64(dx) - want) <= tol)
    assert not off.any(), (np.argwhere(off)[:3], f64(dx)[off][:3], want[off][:3])
    # a group's rows in fp32, groups in 64 bits
    assert (np.abs(f64(dw) - want_w) <= np.abs(d * n).sum(0) * U * (min(d.shape[0], 2 + d.shape[0] / 74) + 3) + np.abs(want_w) * U + 2.0 ** -149).all()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows,cols", SHAPES + [(5000, 520), (2500, 100)])
def test_gradient(b, rows, cols, dtype):
    x, dy, dh = (matrix(rows, cols, dtype, i) for i in range(3))
    w = weight(cols, torch.float32 if cols % 2 else dtype)
    out = b.rms_norm(x, w, 1e-5)
    check_grad(b.rms_norm_grad(dy, x, w, out.rstd), dy, x, w, out.rstd, None)
    check_grad(b.rms_norm_grad(dy, x, w, out.rstd, add=dh), dy, x, w, out.rstd, dh)


def test_gradient_against_differences(b):
    """Along random directions: (loss(x + d) - loss(x - d)) / 2 against the gradient's product with d.  Steps of 2^-6: the third derivative leaves about its square,
    2^-12; sums of 2 x 33 x 700 fp32 outputs, off by 2^-23 of their size each, 2^-23 * 64 / sqrt of their number."""
    x, w, dy = matrix(33, 700, torch.float32, scale=0.5), weight(700, torch.float32), matrix(33, 700, torch.float32, 1)
    out = b.rms_norm(x, w, 0.3)
    dx, dw = b.rms_norm_grad(dy, x, w, out.rstd)
    for seed in range(3):
        d = matrix(33, 700, torch.float32, 10 + seed) * 2.0 ** -6
        d *= x.norm() / matrix(33, 700, torch.float32, 10 + seed).norm()
        e = weight(700, torch.float32, seed) * 2.0 ** -6

        def loss(x, w):
            return float((b.rms_norm(x, w, 0.3).y.double() * dy.double()).sum())

        size = float((dy.double() * out.y.double()).norm())
        got, want = (loss(x + d, w) - loss(x - d, w)) / 2, float((dx.double() * d.double()).sum())
        assert abs(got - want) <= size * 2.0 ** -12 * 4
        got, want = (loss(x, w + e) - loss(x, w - e)) / 2, float((dw.double() * e.double()).sum())
        assert abs(got - want) <= size * 2.0 ** -16


@pytest.mark.parametrize("dtype", DTYPES)
def test_rows_of_zeros_infinities_and_nan(b, dtype):
    for cols in (520, 521, 9000):
        x = matrix(9, cols, dtype)
        w = weight(cols, dtype)
        x[2] = 0
        x[4, 7], x[5, 200], x[6, 0] = float("inf"), float("nan"), float("-inf")
        out = b.rms_norm(x, w, 0.0)
        assert torch.isinf(out.rstd[2]) and torch.isnan(out.y[2]).all()                      # (eps of zero: 0 times infinity)
        assert torch.equal(out.rstd[4], torch.tensor(0.0, device="cuda")) and torch.isnan(out.y[4, 7]) and not out.y[4, 8:].any()
        assert torch.isnan(out.y[5]).all() and torch.isnan(out.rstd[5])
        good = torch.tensor([0, 1, 3, 7, 8], device="cuda")
        assert torch.equal(out.y[good], b.rms_norm(x[good], w, 0.0).y)
        out = b.rms_norm(x, w, 1e-6, forms="both")
        v, t = (b.f8_dequantise(f) for f in out.y)
        assert not v[2].any() and torch.isnan(v[5]).all() and torch.isnan(v[4, :128]).all() and not v[4, 128:].any()
        assert torch.isnan(t).all()                                                          # (each column's block has a NaN of row 5)
        assert torch.equal(v[good], b.f8_dequantise(b.rms_norm(x[good], w, 1e-6, forms="rows").y))


def test_large_and_small_values(b):
    """Squares beyond fp32's range on both ends."""
    for scale in (1e30, 1e-30):
        x, w = matrix(20, 700, torch.float32, scale=scale), weight(700, torch.float32)
        check_norm(b.rms_norm(x, w, 0.0), x, w, 0.0, None, None)
        check_norm(b.rms_norm(x, w, 0.0, forms="both"), x, w, 0.0, None, "both")


def test_no_rows_or_columns(b):
    w = torch.ones(5, device="cuda")
    x = torch.empty(0, 5, device="cuda")
    out = b.rms_norm(x, w, forms="both")
    dx, dw = b.rms_norm_grad(x, x, w, out.rstd)
    assert out.rstd.shape == (0,) and dx.shape == (0, 5) and not dw.any()
    x = torch.empty(3, 0, device="cuda")
    out = b.rms_norm(x, w[:0])
    assert torch.isnan(out.rstd).all() and b.rms_norm_grad(x, x, w[:0], out.rstd)[1].numel() == 0


def test_results_do_not_change(b):
    """Calls of many blocks, twice: the same bits."""
    x, dy, w = matrix(3000, 1600, torch.bfloat16), matrix(3000, 1600, torch.bfloat16, 1), weight(1600, torch.bfloat16)
    out = b.rms_norm(x, w)
    first = b.rms_norm_grad(dy, x, w, out.rstd)
    for _ in range(3):
        assert all(torch.equal(p, q) for p, q in zip(first, b.rms_norm_grad(dy, x, w, out.rstd)))
    # a row's results do not depend on the rows beside it, nor on how many there are
    few = b.rms_norm(x[17:20], w)
    assert torch.equal(few.y, out.y[17:20]) and torch.equal(few.rstd, out.rstd[17:20])


def test_any_leading_dimensions_streams_and_graphs(b):
    x, r, w = matrix(24, 700, torch.bfloat16).view(2, 3, 4, 700), matrix(24, 700, torch.bfloat16, 1).view(2, 3, 4, 700), weight(700, torch.float32)
    want = b.rms_norm(x, w, add=r, forms="rows")
    flat = b.rms_norm(x.view(24, 700), w, add=r.view(24, 700), forms="rows")
    assert want.h.shape == x.shape and want.rstd.shape == (2, 3, 4) and torch.equal(want.y.codes, flat.y.codes) and torch.equal(want.y.scales, flat.y.scales)
    grads = b.rms_norm_grad(x, want.h, w, want.rstd, add=r)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    other = b.rms_norm(x, w, add=r, forms="rows", stream=s)
    others = b.rms_norm_grad(x, other.h, w, other.rstd, add=r, stream=s)
    s.synchronize()
    assert torch.equal(other.y.codes, want.y.codes) and all(torch.equal(p, q) for p, q in zip(grads, others))
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out = b.rms_norm(x, w, add=r, forms="both")
        got = b.rms_norm_grad(x, out.h, w, out.rstd, add=r)
    for seed in range(2):
        x.copy_(matrix(24, 700, torch.bfloat16, 7 + seed).view(x.shape))
        g.replay()
        again = b.rms_norm(x, w, add=r, forms="both")
        assert torch.equal(out.y[0].codes, again.y[0].codes) and torch.equal(out.y[1].codes, again.y[1].codes)
        assert all(torch.equal(p, q) for p, q in zip(got, b.rms_norm_grad(x, again.h, w, again.rstd, add=r)))


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows,cols", [(40, 100), (300, 1600), (37, 1301), (5, 20001)])
def test_in_place(b, rows, cols, dtype):
    """h in x's or the residual's place, y in any of theirs, dx in dy's or the other gradient's."""
    x, r, w = matrix(rows, cols, dtype), matrix(rows, cols, dtype, 1), weight(cols, dtype)
    want = b.rms_norm(x, w, 1e-5, add=r)
    kind = {torch.float32: b.F32, torch.bfloat16: b.BF16, torch.float16: b.F16}[dtype]

    def norm(x, add, h, y):
        rstd = torch.empty(rows, device="cuda")
        rc = b.lib.conef_rms_norm(x.data_ptr(), add.data_ptr() if add is not None else None, w.data_ptr(), kind, kind, rows, cols, cols, cols, 1e-5,
                                  h.data_ptr() if h is not None else None, cols, rstd.data_ptr(), y.data_ptr(), cols, 0, None, None, None, None, None)
        assert rc == b.OK
        return rstd

    for places in (("x", "r"), ("r", "x"), ("x", "x"), ("r", "r")):
        t = dict(x=x.clone(), r=r.clone())
        rstd = norm(t["x"], t["r"], t[places[0]], t[places[1]])
        assert torch.equal(t[places[1]], want.y) and torch.equal(rstd, want.rstd)
        if places[0] != places[1]:
            assert torch.equal(t[places[0]], want.h)
    alone = x.clone()
    norm(alone, None, None, alone)
    assert torch.equal(alone, b.rms_norm(x, w, 1e-5).y)
    dx, dw = b.rms_norm_grad(r, want.h, w, want.rstd, add=x)
    for place in ("dy", "add"):
        t, got = dict(dy=r.clone(), add=x.clone()), torch.empty(cols, device="cuda")
        size = C.c_size_t()
        assert b.lib.conef_rms_norm_grad_bytes(rows, cols, C.byref(size)) == b.OK
        space = torch.empty(size.value, dtype=torch.uint8, device="cuda")
        rc = b.lib.conef_rms_norm_grad(t["dy"].data_ptr(), want.h.data_ptr(), w.data_ptr(), want.rstd.data_ptr(), t["add"].data_ptr(), kind, kind, rows, cols, cols, cols, cols,
                                       t[place].data_ptr(), cols, got.data_ptr(), space.data_ptr(), size.value, None)
        assert rc == b.OK
        assert torch.equal(t[place], dx) and torch.equal(got, dw)


def test_in_an_autograd_function(b):
    class Norm(torch.autograd.Function):
        @staticmethod
        def forward(ctx, x, w, add):
            y, h, rstd = b.rms_norm(x, w, 1e-5, add=add)
            ctx.save_for_backward(h, w, rstd)
            return y, h

        @staticmethod
        def backward(ctx, dy, dh):
            h, w, rstd = ctx.saved_tensors
            dx, dw = b.rms_norm_grad(dy.contiguous(), h, w, rstd, add=dh.contiguous())
            return dx, dw, dx

    x, r, w = (t.requires_grad_() for t in (matrix(9, 130, torch.float32), matrix(9, 130, torch.float32, 1), weight(130, torch.float32)))
    with pytest.raises(b.ConEFError):
        b.rms_norm(x, w)
    y, h = Norm.apply(x, w, r)
    (y.square().sum() + h.sum()).backward()
    xd, rd, wd = (t.detach().double().requires_grad_() for t in (x, r, w))
    hd = xd + rd
    ((hd * torch.rsqrt(hd.square().mean(1, keepdim=True) + 1e-5) * wd).square().sum() + hd.sum()).backward()
    for t, d in ((x, xd), (r, rd), (w, wd)):
        assert (t.grad.double() - d.grad).norm() <= 1e-5 * d.grad.norm()


def test_refusals(b):
    x, w = matrix(4, 8, torch.bfloat16), weight(8, torch.bfloat16)
    out = b.rms_norm(x, w)
    bad = [lambda: b.rms_norm(x, w[:7]), lambda: b.rms_norm(x, w.half()), lambda: b.rms_norm(x, w.cpu()), lambda: b.rms_norm(x, w, add=x[:3]),
           lambda: b.rms_norm(x, w, add=x.float()), lambda: b.rms_norm(x.t(), w[:4]), lambda: b.rms_norm(x, w, forms="all"), lambda: b.rms_norm(x, w, forms="rows", kind="x"),
           lambda: b.rms_norm(x, w, -1.0), lambda: b.rms_norm(x, w, float("nan")), lambda: b.rms_norm_grad(x, x, w, out.rstd[:3]),
           lambda: b.rms_norm_grad(x, x.float(), w, out.rstd), lambda: b.rms_norm_grad(x, x, w, out.rstd.double()), lambda: b.rms_norm_grad(x, x[:, :7], w, out.rstd),
           lambda: b.rms_norm_grad(x, x, w, out.rstd, add=x[:2]), lambda: b.rms_norm(x, w.float().requires_grad_())]
    for call in bad:
        with pytest.raises(b.ConEFError) as e:
            call()
        assert e.value.code == b.ERR_INVALID_ARG

"""Dropout, microscaled 4-bit floats and the step on them where offsets pass 32 bits, and where blocks are more than 32 bits count: rows and columns
picked from the whole, against the plain statement in 64 bits."""
import numpy as np
import pytest
import torch

from oracle import mx4_oracle as mo

pytestmark = pytest.mark.gpu
SEED = (5, 1, 2, 3)
ROWS, COLS = 66000, 65540   # 4.3e9 elements, 8.7 GB in 16 bits


@pytest.fixture(scope="module")
def b():
    from paper_2312_08538_b200 import binding
    yield binding
    torch.cuda.empty_cache()


def numbers(r, c, cols, which):
    """The numbers of rows r and columns c of a matrix of `cols` columns."""
    r, c = np.asarray(r, np.uint64)[:, None], np.asarray(c, np.uint64)[None, :]
    with np.errstate(over="ignore"):
        j = np.uint64(2) * (r * np.uint64((cols + 3) // 4) + c // np.uint64(4)) + np.uint64(which)
        z = np.uint64(mo.stream(*SEED)) + np.uint64(mo._G) * (j + np.uint64(1))
        z = (z ^ (z >> np.uint64(30))) * np.uint64(0xBF58476D1CE4E5B9)
        z = (z ^ (z >> np.uint64(27))) * np.uint64(0x94D049BB133111EB)
        z = z ^ (z >> np.uint64(31))
    return ((z >> (np.uint64(16) * (c % np.uint64(4)))) & np.uint64(0xFFFF)).astype(np.int64)


def test_numbers_are_those_of_the_oracle():
    assert np.array_equal(numbers(range(5), range(7), 7, 1), mo.numbers(*SEED, 5, 7, 1))


@pytest.fixture(scope="module")
def x():
    gen = torch.Generator(device="cuda")
    gen.manual_seed(1)
    m = torch.empty(ROWS, COLS, dtype=torch.bfloat16, device="cuda")
    m.copy_(torch.randn(1, COLS, generator=gen, device="cuda"))
    m.mul_(torch.exp2((torch.arange(ROWS, device="cuda") % 7 - 3).float()).to(torch.bfloat16)[:, None])   # (exact)
    return m


PICK = [0, 1, 65531, 65532, 65534, 65535, 65536, 65997, 65999]


def dropped(values, u, p):
    f = int(np.rint(p * 65536))
    return np.where(u >= f, values * np.float32(65536.0 / (65536 - f)), np.float32(0))


@pytest.mark.parametrize("front,cols", [(0, COLS), (1, 65537)])   # one array, and rows of a wider one
def test_dropout(b, x, front, cols):
    v = x[:, front:front + cols]
    y = b.dropout(v, 0.25, b.Draw(*SEED))
    u = numbers(PICK, range(cols), cols, mo.DROPOUT)
    want = torch.from_numpy(dropped(v[PICK].float().cpu().numpy(), u, 0.25)).to(torch.bfloat16)
    assert torch.equal(y[PICK].cpu(), want)


def form_rows(form, pick):
    """Codes and scale bytes of some rows of a form."""
    nb, tiles = (form.cols + 31) // 32, (form.cols + 127) // 128
    raw = form.codes.view(form.rows, nb * 16)[pick].cpu().numpy()
    codes = np.stack([raw & 15, raw >> 4], -1).reshape(len(pick), nb * 32)
    r, blk = np.asarray(pick, np.int64)[:, None], np.arange(nb)[None, :]
    at = ((r // 128) * tiles + blk // 4) * 512 + (r % 32) * 16 + (r % 128) // 32 * 4 + blk % 4
    assert not codes[:, form.cols:].any()
    return codes[:, :form.cols], form.scales[torch.from_numpy(at).cuda()].cpu().numpy()


def test_quantise_and_values(b, x):
    how = dict(stochastic=True, p=0.25, draw=b.Draw(*SEED))
    a, t = b.mx4_quantise(x, forms="both", **how)
    alone = b.mx4_quantise(x, **how)
    assert torch.equal(alone.codes, a.codes) and torch.equal(alone.scales, a.scales)
    del alone
    for form, pick, other in ((a, PICK, range(COLS)), (t, [0, 3, 32768, 65535, 65536, 65539], range(ROWS))):
        r, c = (pick, other) if form is a else (other, pick)
        v = (x[pick] if form is a else x[:, pick]).float().cpu().numpy()
        v = dropped(v, numbers(r, c, COLS, mo.DROPOUT), 0.25).astype(np.float64)
        u = numbers(r, c, COLS, mo.ROUNDING)
        want = mo.encode(v, u) if form is a else mo.encode(v.T.copy(), u.T.copy())
        got = form_rows(form, pick)
        assert np.array_equal(got[1], want[1]) and np.array_equal(got[0], want[0])
        values = b.mx4_dequantise(form)
        assert np.array_equal(values[pick].cpu().numpy(), mo.decode(*want).astype(np.float32))
        del values


def test_product(b, x):
    k = 64
    a, w = b.mx4_quantise(x[:, :k]), b.mx4_quantise(x[:COLS, k:2 * k])
    out = b.mx4_matmul(a, w)
    va, vw = mo.decode(*form_rows(a, PICK)), mo.decode(*form_rows(w, list(range(COLS))))
    want, size = va @ vw.T, np.abs(va) @ np.abs(vw).T
    tol = k * 2.0 ** -23 * size + np.abs(want) * 2.0 ** -8 * 1.001 + 1e-30   # (sums in fp32, one rounding)
    assert (np.abs(out[PICK].double().cpu().numpy() - want) <= tol).all()


def test_more_blocks_than_32_bits_count(b):
    """A column of 2^30 + 300 rows: four (padded) blocks to each, so several launches."""
    rows = (1 << 30) + 300
    v = torch.empty(rows, 1, dtype=torch.bfloat16, device="cuda")
    v.copy_((torch.arange(rows, device="cuda") % 251 - 125).to(torch.bfloat16)[:, None])
    a = b.mx4_quantise(v, stochastic=True, p=0.25, draw=b.Draw(*SEED))
    pick = [0, 1, 127, 128, (1 << 30) - 1025, (1 << 30) - 1024, (1 << 30) - 1023, (1 << 30) - 1, 1 << 30, rows - 1]
    val = dropped(v[pick].float().cpu().numpy(), numbers(pick, [0], 1, mo.DROPOUT), 0.25).astype(np.float64)
    want = mo.encode(val, numbers(pick, [0], 1, mo.ROUNDING))
    got = form_rows(a, pick)
    assert np.array_equal(got[1], want[1]) and np.array_equal(got[0], want[0])
    assert int(a.scales[-512:].count_nonzero()) <= 128       # rows and blocks that do not exist
    y = b.mx4_dequantise(a)
    assert np.array_equal(y[pick].cpu().numpy(), mo.decode(*want).astype(np.float32))
    y = b.dropout(v, 0.25, b.Draw(*SEED))
    assert torch.equal(y[pick].cpu(), torch.from_numpy(dropped(v[pick].float().cpu().numpy(), numbers(pick, [0], 1, mo.DROPOUT), 0.25)).to(torch.bfloat16))


@pytest.mark.parametrize("kind", ["mx4", "mx4-stochastic"])
def test_a_tensor_of_more_than_2_to_31_elements(b, kind):
    """Its state is the form of its rows (their width being whole blocks), but for what was sent."""
    rows, cols = 34000, 65536
    eng = b.ConEF([(rows, cols, 1)], 1, dict(kind="randblock", k_num=1, k_den=rows * cols, seed=9), dict(kind=kind, seed=SEED[0]), 1.0)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(3)
    g = torch.empty(rows * cols, device="cuda").normal_(generator=gen)
    eng.full_step(SEED[3], [g])
    at = int(eng.indices(0)[0].item()) & 0xFFFFFFFF
    g[at] = 0.0
    # the step's worker is 0, its tensor 0
    want = b.mx4_dequantise(b.mx4_quantise(g.view(rows, cols), stochastic=kind == "mx4-stochastic", draw=b.Draw(SEED[0], 0, 0, SEED[3])))
    assert torch.equal(eng.decompress_error(0).view(rows, cols), want)

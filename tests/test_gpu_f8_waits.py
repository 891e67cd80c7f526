"""Products of 8-bit forms and orthogonalised updates whose thread blocks wait for loads that never come: each wait runs out after a millisecond, the kernel ends, the
count tells, what was not computed is NaN and the rest is right, and so is the next one."""
import pytest
import torch

from tests.test_gpu_f8 import DTYPES, b, matrix  # noqa: F401  (b: a fixture)
from tests.test_gpu_orthogonalise import update

pytestmark = pytest.mark.gpu


@pytest.fixture
def short_waits(b):
    yield lambda loads, second=-1: b.mx4_set_waits(1e-3, loads, second)
    b.mx4_set_waits()


def check(b, short_waits, shape, dtype, loads, second=-1):
    m, n, k = shape
    a, c = b.f8_quantise(matrix(m, k, torch.bfloat16)), b.f8_quantise(matrix(n, k, torch.bfloat16, 1, 0.02), kind="e5m2")
    want = b.f8_matmul(a, c, dtype)
    before = b.f8_timeouts()
    short_waits(loads, second)
    got = b.f8_matmul(a, c, dtype)
    b.mx4_set_waits()
    after = b.f8_timeouts()
    assert after > before
    lost = torch.isnan(got)
    assert lost.any() and torch.equal(torch.where(lost, want, got), want)
    assert all(torch.equal(b.f8_matmul(a, c, dtype), want) for _ in range(3))
    assert b.f8_timeouts() == after
    return int(lost.sum()), m * n


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("loads", [0, 1, 5, 12])
def test_blocks_on_their_own(b, short_waits, loads, dtype):
    """A tile and thirteen stages to each: nothing is computed."""
    lost, all_of_them = check(b, short_waits, (1000, 1000, 1600), dtype, loads)
    assert lost == all_of_them


@pytest.mark.parametrize("shape,loads", [((40000, 64, 1600), 13), ((40000, 64, 1600), 30), ((40001, 187, 1603), 17)])
def test_blocks_with_several_tiles(b, short_waits, shape, loads):
    """The first tiles are computed."""
    lost, all_of_them = check(b, short_waits, shape, torch.bfloat16, loads)
    assert lost < all_of_them


@pytest.mark.parametrize("loads,second", [(0, 0), (0, -1), (-1, 0), (3, -1), (-1, 3), (2, 4), (4, 2), (20, 20), (21, -1), (-1, 22)])
def test_pairs_that_bring_different_numbers_of_stages(b, short_waits, loads, second):
    lost, all_of_them = check(b, short_waits, (8192, 6400, 1600), torch.bfloat16, loads, second)
    assert (lost == all_of_them) == (min(x for x in (loads, second) if x >= 0) < 13)


@pytest.mark.parametrize("rows,cols,batch", [(100, 300, 1), (600, 200, 3), (1600, 1600, 1), (700, 2500, 3)])
@pytest.mark.parametrize("loads,second", [(0, 0), (1, 1), (0, -1), (-1, 0), (3, 5), (6, 2), (7, 7)])   # (blocks that share a tile along its rows bring six)
def test_orthogonalise(b, short_waits, rows, cols, batch, loads, second):
    """Few steps, so that the waits of all launches last a second at most; a product that lacks a tile leaves NaN in the next ones' sums."""
    x = torch.stack([update(rows, cols, torch.bfloat16, i) for i in range(batch)])
    want = b.orthogonalise(x, steps=2)
    before = b.orthogonalise_timeouts()
    short_waits(loads, second)
    got = b.orthogonalise(x, steps=2)
    b.mx4_set_waits()
    after = b.orthogonalise_timeouts()
    lost = torch.isnan(got)
    assert after > before or loads < 0   # (blocks on their own have no second one)
    assert bool(lost.any()) == (after > before)
    assert torch.equal(torch.where(lost, want, got), want)
    assert all(torch.equal(b.orthogonalise(x, steps=2), want) for _ in range(3))
    assert b.orthogonalise_timeouts() == after


@pytest.mark.parametrize("shape,loads", [((100, 1600, 6400), 0), ((100, 1600, 6400), 5), ((200, 130, 20000), 17), ((256, 256, 33001), 6), ((768, 768, 8192), 31)])
def test_blocks_that_share_a_tile_along_k(b, short_waits, shape, loads):
    """Nothing is computed, also where the last blocks of tiles, which have fewer stages (11 of 13, 17 of 20), have all of theirs."""
    lost, all_of_them = check(b, short_waits, shape, torch.bfloat16, loads)
    assert lost == all_of_them


@pytest.mark.parametrize("rows,cols,loads", [(100, 4000, 0), (100, 4000, 3), (100, 4000, 13), (300, 5000, 0), (300, 5000, 3), (300, 5000, 9)])
def test_orthogonalise_long_rows(b, short_waits, rows, cols, loads):
    """Blocks that share a tile along its rows: of 4000 16 half stages each (the last ones 14), of 5000, from 256 rows on the hi parts alone, 10 of 79 stages (the last ones,
    which have all of theirs with loads = 9, 9): nothing is computed."""
    x = update(rows, cols, torch.bfloat16)
    want = b.orthogonalise(x, steps=2)
    before = b.orthogonalise_timeouts()
    short_waits(loads)
    got = b.orthogonalise(x, steps=2)
    b.mx4_set_waits()
    assert b.orthogonalise_timeouts() > before and torch.isnan(got).all()
    assert all(torch.equal(b.orthogonalise(x, steps=2), want) for _ in range(3))

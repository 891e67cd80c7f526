"""Products of microscaled 4-bit floats whose thread blocks wait for loads that never come: each wait runs out after a millisecond, the kernel ends, the count
tells, what was not computed is NaN and the rest is right, and so is the next product."""
import pytest
import torch

from tests.test_gpu_mx4 import DTYPES, b, matrix  # noqa: F401  (b: a fixture)

pytestmark = pytest.mark.gpu


@pytest.fixture
def short_waits(b):
    yield lambda loads, second=-1: b.mx4_set_waits(1e-3, loads, second)
    b.mx4_set_waits()


def check(b, short_waits, shape, dtype, loads, second=-1):
    m, n, k = shape
    a, c = b.mx4_quantise(matrix(m, k, torch.bfloat16)), b.mx4_quantise(matrix(n, k, torch.bfloat16, 1, 0.02))
    want = b.mx4_matmul(a, c, dtype=dtype)
    before = b.mx4_timeouts()
    short_waits(loads, second)
    got = b.mx4_matmul(a, c, dtype=dtype)
    b.mx4_set_waits()
    after = b.mx4_timeouts()
    assert after > before
    lost = torch.isnan(got)
    assert lost.any() and torch.equal(torch.where(lost, want, got), want)
    assert all(torch.equal(b.mx4_matmul(a, c, dtype=dtype), want) for _ in range(3))
    assert b.mx4_timeouts() == after
    return int(lost.sum()), m * n


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("loads", [0, 1, 4, 6])
def test_blocks_on_their_own(b, short_waits, loads, dtype):
    """A tile of 64 columns and seven stages to each: nothing is computed."""
    lost, all_of_them = check(b, short_waits, (1000, 1000, 1600), dtype, loads)
    assert lost == all_of_them


@pytest.mark.parametrize("shape,loads", [((40000, 64, 1600), 7), ((40000, 64, 1600), 16), ((40001, 187, 1603), 9), ((3352, 4048, 2100), 12), ((3353, 4043, 2100), 20)])
def test_blocks_with_several_tiles(b, short_waits, shape, loads):
    """64, 192 and 256 columns; the first tiles are computed."""
    lost, all_of_them = check(b, short_waits, shape, torch.bfloat16, loads)
    assert lost < all_of_them


@pytest.mark.parametrize("shape", [(8192, 6400, 1600), (3330, 4113, 2100), (4120, 3280, 2100)])
@pytest.mark.parametrize("loads,second", [(0, 0), (0, -1), (-1, 0), (3, 3), (3, -1), (-1, 3), (2, 4), (4, 2), (11, 11), (12, -1), (-1, 13), (20, 18)])
def test_pairs_that_bring_different_numbers_of_stages(b, short_waits, shape, loads, second):
    """192 columns, with and without tiled outputs, and 256: either block of a pair stops, or both at different stages."""
    lost, all_of_them = check(b, short_waits, shape, torch.bfloat16, loads, second)
    assert (lost == all_of_them) == (min(x for x in (loads, second) if x >= 0) < (shape[2] + 255) // 256)


def test_nothing_runs_out_otherwise(b):
    assert b.mx4_timeouts() == b.mx4_timeouts(torch.device("cuda", torch.cuda.current_device())) == b.mx4_timeouts(stream=torch.cuda.Stream())
    before = b.mx4_timeouts()
    a, c = b.mx4_quantise(matrix(3330, 2100, torch.bfloat16)), b.mx4_quantise(matrix(4113, 2100, torch.bfloat16, 1))
    for _ in range(5):
        assert not torch.isnan(b.mx4_matmul(a, c)).any()
    assert b.mx4_timeouts() == before

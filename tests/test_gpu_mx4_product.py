"""Products of microscaled 4-bit floats: sizes that take every kind of tile, sums over more than 2^30 elements, two products at once."""
import pytest
import torch

from tests.test_gpu_mx4 import b  # noqa: F401  (a fixture)

pytestmark = pytest.mark.gpu


# ------------------------------------------------------------------ long sums

@pytest.mark.parametrize("rows,k", [(1, (1 << 30) + 1000), (2, (1 << 30) + 1000), (1, (1 << 31) - 1)])
def test_sums_over_more_than_2_to_30_elements(b, rows, k):
    """Rows that are zero but for a block at the beginning and one behind element 2^30, whose scales differ."""
    blocks, tiles, far = (k + 31) // 32, (k + 127) // 128, (k - 100) // 32

    def form(scale, far_scale, values):
        codes = torch.zeros(rows, blocks * 16, dtype=torch.uint8, device="cuda")
        scales = torch.zeros(tiles * 512, dtype=torch.uint8, device="cuda")
        for r in range(rows):
            for block, byte in ((0, scale), (far, far_scale)):
                codes[r, block * 16:block * 16 + 16] = values[r]
                scales[(block // 4) * 512 + r * 16 + block % 4] = byte
        return b.MX4(rows, k, codes, scales)

    a, c = form(127, 130, [0x22, 0x44]), form(127, 126, [0x22, 0x55])       # 1, 2 by 1, 3; scales 1, 8 by 1, 1/2
    want = torch.tensor([[32 + 32 * 8 * 0.5, (32 + 32 * 8 * 0.5) * 3], [(32 + 32 * 8 * 0.5) * 2, (32 + 32 * 8 * 0.5) * 6]])[:rows, :rows]
    assert torch.equal(b.mx4_matmul(a, c, dtype=torch.float32).cpu(), want)

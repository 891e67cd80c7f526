"""Products of microscaled 4-bit floats: sizes that take every kind of tile, sums over more than 2^30 elements, two products at once."""
import pytest
import torch

from tests.test_gpu_mx4 import DTYPES, EPS, TINY, b, matrix  # noqa: F401  (b: a fixture)

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


# ------------------------------------------------------------------ kinds of tiles

PER_STEP, PER_TILE = ((45, 52, 67, 88), (0, 48, 60, 73)), (700, 970, 1240, 2450)


def kind_of(m, n, k):
    """The library's choice (mm_choice in conef_mx4mm.cu): (pair, columns, tiles per CTA or pair at most)."""
    best = None
    for pair in (0, 1):
        for i in range(pair, 4):
            tiles = -(-m // (256 if pair else 128)) * -(-n // (64 * (i + 1)))
            waves = -(-tiles // (74 if pair else 148))
            cost = waves * (-(-k // 64) * PER_STEP[pair][i] + PER_TILE[i]) + pair * 1000
            if best is None or cost < best[0]:
                best = cost, (pair, 64 * (i + 1), waves)
    return best[1]


# two or more tiles to each CTA or pair, and more stages than a ring has; outputs by tiled copies where n is a multiple of 8, else by elements
KINDS = [((40000, 64, 1600), (0, 64, 3)), ((40001, 61, 651), (0, 64, 3)), ((40000, 128, 1600), (0, 128, 3)), ((40001, 123, 1603), (0, 128, 3)),
         ((40000, 192, 1600), (0, 192, 3)), ((40001, 187, 1603), (0, 192, 3)), ((3352, 4048, 2100), (0, 256, 3)), ((3353, 4043, 2100), (0, 256, 3)),
         ((4797, 776, 8192), (1, 128, 2)), ((5639, 1729, 4100), (1, 128, 5)), ((8192, 6400, 1600), (1, 192, 15)), ((3330, 4113, 2100), (1, 192, 5)),
         ((6400, 1600, 8192), (1, 256, 3)), ((4120, 3280, 2100), (1, 256, 3)), ((4120, 3273, 2100), (1, 256, 3)), ((1111, 2601, 651), (0, 192, 1))]


def forms(b, m, n, k):
    return b.mx4_quantise(matrix(m, k, torch.bfloat16)), b.mx4_quantise(matrix(n, k, torch.bfloat16, 1, 0.02))


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("shape,kind", KINDS)
def test_every_kind_of_tile(b, shape, kind, dtype):
    """Into the columns of a wider matrix, through the C interface.  Products are exact in fp32; each of the k sums is off by 2^-23 of the sum of sizes at
    most, and the result is rounded once (as in check_product)."""
    m, n, k = shape
    assert kind_of(m, n, k) == kind
    a, c = forms(b, m, n, k)
    wide = torch.full((m + 2, n + 8), 7.0, dtype=dtype, device="cuda")
    code = {torch.float32: b.F32, torch.bfloat16: b.BF16, torch.float16: b.F16}[dtype]
    at = wide.data_ptr() + (n + 8) * wide.element_size()
    assert b.lib.conef_mx4_matmul(a.codes.data_ptr(), a.scales.data_ptr(), m, c.codes.data_ptr(), c.scales.data_ptr(), n, k, at, code, n + 8, b._stream_handle(None)) == b.OK
    va, vc = b.mx4_dequantise(a).double(), b.mx4_dequantise(c).double()
    want, size = va @ vc.t(), va.abs() @ vc.abs().t()
    got = wide[1:-1, :n].double()
    off = ~((got - want).abs() <= k * 2.0 ** -23 * size + want.abs() * EPS[dtype] * 1.001 + TINY[dtype])
    assert not off.any(), (off.nonzero()[:3], got[off][:3], want[off][:3])
    assert torch.equal(b.mx4_matmul(a, c, dtype=dtype), wide[1:-1, :n])
    wide[1:-1, :n] = 7.0
    assert (wide == 7).all()


def test_pairs_on_two_streams_at_once(b):
    """Pairs of CTAs of two products without an order between them, and of a replayed graph: each takes all of two SMs' tensor memory."""
    shapes = [(3330, 4113, 2100), (4120, 3280, 2100), (4797, 776, 8192)]
    jobs = [forms(b, *s) for s in shapes]
    want = [b.mx4_matmul(*j) for j in jobs]
    before = b.mx4_timeouts()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = [b.mx4_matmul(*jobs[2]) for _ in range(4)]
    streams = [torch.cuda.Stream() for _ in jobs]
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(20):
        for i in range(2):
            got[i].append(b.mx4_matmul(*jobs[i], stream=streams[i]))
        with torch.cuda.stream(streams[2]):
            graph.replay()
    torch.cuda.synchronize()
    for w, runs in zip(want, got + [captured]):
        assert all(torch.equal(w, r) for r in runs)
    assert b.mx4_timeouts() == before

"""The 8-bit operators at the ends of their ranges and on the tile widths, splits
and grids that large sizes take: equality with whole-number sums formed in 64
bits, codes within half a step (as in the tests of ordinary sizes)."""

import pytest
import torch

import test_gpu_q8 as ordinary
from q8_plans import PLANS, row_stride
from test_gpu_q8 import expected, padded, product

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def lib():
    from paper_2607_14672_gb300 import build, dstd
    build.build()
    dstd.load()
    assert dstd.device_status(clear=True) == 0
    yield
    assert dstd.device_status(clear=True) == 0


def test_quantize_row_of_the_longest_length():
    """One row of 2^31 - 1 columns: its codes at both ends and between, zeros elsewhere, nothing around it."""
    from paper_2607_14672_gb300 import dstd
    K, around = 2 ** 31 - 1, 4096
    at = [0, 1, 255, 256, 2 ** 30, K - 257, K - 256, K - 255, K - 2, K - 1]
    want = [127, -127, 64, 3, -5, 100, -100, 17, 1, -64]      # whole numbers, the largest 127: the codes themselves
    x = torch.zeros(1, K, dtype=torch.bfloat16, device="cuda")
    x[0, at] = torch.tensor(want, dtype=torch.bfloat16, device="cuda")
    room = torch.full((K + 2 * around,), 55, dtype=torch.int8, device="cuda")
    q, scale = room[around:around + K].view(1, K), torch.empty(1, device="cuda")
    dstd.quantize_rows(x, q, scale)
    torch.cuda.synchronize()
    assert scale.item() == 1.0
    assert q[0, at].tolist() == want
    assert sum(int(part.count_nonzero()) for part in q[0].split(1 << 28)) == len(at)
    assert (room[:around] == 55).all() and (room[around + K:] == 55).all()


@pytest.mark.parametrize("i", range(len(PLANS)))
def test_int8_matmul_tile_widths_and_splits(i):
    """Every tile width of the tensor-core form, in one piece, cut along K, and both, from either side."""
    T, N, K, nt, form, exchanged = PLANS[i]
    dtype = (torch.float32, torch.bfloat16, torch.float16)[i % 3]
    g = torch.Generator(device="cuda").manual_seed(i)
    x, w = (padded(torch.randint(-128, 128, (R, K), generator=g, device="cuda"), row_stride(K) - K, torch.int8)
            for R in (T, N))
    sx = torch.rand(T, generator=g, device="cuda") + 0.01
    sw = torch.rand(N, generator=g, device="cuda") * 0.01 + 1e-5
    out = torch.full((T, N), 77.0, dtype=dtype, device="cuda")
    product(x, sx, w, sw, out)
    assert torch.equal(out, expected(x, sx, w, sw, dtype))


# more inputs than one block of the token writer takes (4096); layers whose product runs with the sides exchanged
@pytest.mark.parametrize("B,N_in,N_out,M", [(2, 5000, 60, 16), (2, 9001, 40, 32), (2, 16384, 50, 8), (64, 300, 21, 32),
                                            (128, 2000, 40, 32), (64, 1500, 130, 32)])
def test_dense_fwd_q8_of_other_sizes(B, N_in, N_out, M):
    """The layer against the oracle on the public quantiser's codes, with the tolerances of the ordinary sizes."""
    ordinary.test_dense_fwd_q8(B, N_in, N_out, M)

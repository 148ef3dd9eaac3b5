"""The 8-bit operators at the ends of their ranges and on the tile widths, splits
and grids that large sizes take: equality with whole-number sums formed in 64
bits, codes within half a step (as in the tests of ordinary sizes)."""

import pytest
import torch

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

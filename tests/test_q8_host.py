"""Host code of the 8-bit and clipping calls, without a GPU: what is refused at
the ends of the ranges, and what is launched (through a runtime that runs
nothing, see fake_cuda.cpp)."""

import ctypes

import pytest

import fake_cuda

pytestmark = pytest.mark.skipif(fake_cuda.compiler() is None, reason="no C++ compiler")

P = ctypes.c_void_p(256)
OK, UNSUPPORTED = 0, -2


@pytest.fixture(scope="module")
def loaded():
    try:
        from paper_2607_14672_gb300 import build
        build.nvcc_path()
    except RuntimeError:
        pytest.skip("nvcc not available")
    return fake_cuda.load()


@pytest.fixture
def lib(loaded):
    loaded.fake_reset()
    return loaded


def product(lib, T, N, K, out_type=0, ld_out=None, x=P, w=P, ld=None, bytes=1 << 62):
    ld = ld or (K + 15) // 16 * 16
    return lib.dstd_int8_matmul(x, ld, P, w, ld, P, T, N, K, P, out_type, ld_out or N, P, bytes, None)


TOP = 2 ** 31 - 1


@pytest.mark.parametrize("T,N", [(TOP, 1), (TOP - 254, 8), (TOP, 32), (9, TOP), (40, TOP - 254), (TOP, TOP)])
def test_sizes_whose_tiles_pass_32_bits_are_refused(lib, T, N):
    """Tile counts of these were formed past 32 bits: workspaces of 2^64 bytes and plans of no tiles."""
    for size in (lib.dstd_int8_matmul_workspace_bytes, lib.dstd_int8_matmul_aligned_workspace_bytes):
        assert size(T, N, 16) == 0
    assert product(lib, T, N, 16, bytes=(1 << 64) - 1) == UNSUPPORTED
    assert lib.fake_launches() == 0


@pytest.mark.parametrize("T,N", [(TOP - 255, 1), (9, TOP - 255), (8, TOP), (1, TOP)])
def test_the_largest_sizes_are_taken(lib, T, N):
    need = lib.dstd_int8_matmul_workspace_bytes(T, N, 16)
    # at most both sides' rows in 16 bits and the sums of 76 tiles
    assert 0 < need <= 2 * 16 * (T + N) + 76 * (64 + 1024 * 192) + 512
    assert product(lib, T, N, 16, bytes=need) == OK
    names = [l[0] for l in fake_cuda.launches(lib)]
    assert len(names) == 1 and "k_q8_few" in names[0] or "k_q8_prep" in names[0] and "k_q8_tc" in names[1]

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


def big(lib):
    """A product of the tensor-core form: its result, and the launches since."""
    lib.fake_keep_arg2_of(b"k_q8_tc")
    before = lib.fake_launches()
    code = product(lib, 4096, 4096, 4096)
    names = fake_cuda.launches(lib)[before:]
    assert code != OK or any("k_q8_tc" in n[0] for n in names)
    return code, names


def test_product_on_another_device(loaded):
    """The grant of shared memory and the pairs that fit belong to a device."""
    lib = fake_cuda.load()                            # a library that has launched nothing yet
    lib.fake_reset()
    for device in (0, 1, 2, 0):
        lib.fake_device(device)
        code, names = big(lib)
        assert code == OK
        assert all(n[3] == device for n in names)
        # at most the pairs of SMs that this device has room for (fake_cuda.cpp: 76, 76, 50)
        assert names[-1][1] <= 2 * (50 if device == 2 else 76)
        assert product(lib, 2, 64, 64) == OK


@pytest.mark.parametrize("what", ["fake_refuse_attributes", "fake_refuse_occupancy"])
def test_product_after_a_failure(loaded, what):
    """A runtime call that fails once fails that product, and no later one."""
    lib = fake_cuda.load()
    lib.fake_reset()
    getattr(lib, what)(1)
    assert big(lib)[0] != OK
    assert big(lib)[0] == OK


def tensor_list(sizes):
    k = len(sizes)
    return (ctypes.c_void_p * k)(*[256] * k), (ctypes.c_int64 * k)(*sizes), (ctypes.c_int32 * k)(*[0] * k)


def step(lib, sizes):
    g, n, ty = tensor_list(sizes)
    before = lib.fake_launches()
    code = lib.dstd_adamw_clip(len(sizes), g, g, g, g, n, ty, 1e-3, 0.9, 0.999, 1e-8, 1e-2, 1.0, P, None, P, P,
                               lib.dstd_grad_norm_workspace_bytes(len(sizes), n), None)
    return code, fake_cuda.launches(lib)[before:]


def test_step_on_another_device(loaded):
    """The blocks of the cooperative launch are those that fit on the present device."""
    lib = fake_cuda.load()
    lib.fake_reset()
    for device, fit in ((0, 608), (2, 300), (1, 608)):
        lib.fake_device(device)
        code, names = step(lib, [10000000])
        assert code == OK and len(names) == 1 and "k_clip_once" in names[0][0]
        assert 0.9 * fit < names[0][1] <= fit and lib.fake_cooperative(lib.fake_launches() - 1) == 1


def test_step_after_a_failure(loaded):
    lib = fake_cuda.load()
    lib.fake_reset()
    lib.fake_refuse_occupancy(1)
    assert step(lib, [1000])[0] != OK
    assert step(lib, [1000])[0] == OK

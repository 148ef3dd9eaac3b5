"""Host code of the 8-bit and clipping calls, without a GPU: what is refused at
the ends of the ranges, and what is launched (through a runtime that runs
nothing, see fake_cuda.cpp)."""

import ctypes
import struct

import pytest

import fake_cuda
from q8_plans import PLANS, row_stride

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


def test_timing_counts_every_launch(lib):
    """The launches that the timing of a kind reports are those that were made."""
    def counted(call):
        lib.dstd_timing_enable(1)
        before = lib.fake_launches()
        assert call() == OK
        ms, n, total = ctypes.c_float(), ctypes.c_int64(), 0
        for k in range(lib.dstd_kernel_kind_count()):
            assert lib.dstd_timing_read(k, ctypes.byref(ms), ctypes.byref(n)) == OK
            total += n.value
        lib.dstd_timing_enable(0)
        return total, lib.fake_launches() - before

    def clip(sizes):
        g, n, ty = tensor_list(sizes)
        return lib.dstd_clip_grads(len(sizes), g, g, n, ty, 1.0, P, P, lib.dstd_grad_norm_workspace_bytes(len(sizes), n), None)

    def norm(sizes):
        g, n, ty = tensor_list(sizes)
        return lib.dstd_grad_norm(len(sizes), g, n, ty, P, None, P, lib.dstd_grad_norm_workspace_bytes(len(sizes), n), None)

    made = []
    for call in (lambda: product(lib, 0, 64, 64), lambda: product(lib, 2, 64, 64), lambda: product(lib, 4096, 4096, 4096),
                 lambda: lib.dstd_quantize_rows(P, 0, 0, 16, 16, P, 16, P, None, 0, None),
                 lambda: lib.dstd_quantize_rows(P, 0, 3, 16, 16, P, 16, P, None, 0, None),
                 lambda: norm([100]), lambda: norm([100] * 600), lambda: clip([100]), lambda: clip([1 << 20]),
                 lambda: clip([100] * 600), lambda: step(lib, [1 << 20])[0], lambda: step(lib, [1 << 25])[0],
                 lambda: step(lib, [10] * 1100)[0]):
        total, launched = counted(call)
        assert total == launched
        made.append(launched)
    assert made == [0, 1, 2, 0, 1, 1, 2, 1, 2, 4, 1, 2, 6]


@pytest.mark.parametrize("sizes", [(64,), (1 << 24,), ((1 << 24) - 7, 7), ((1 << 24) - 7, 8), (1 << 26, 5), (3,) * 512,
                                   (3,) * 513, (3,) * 1025])
def test_networks_count_the_launches_of_a_clipped_step(lib, sizes):
    """DenseNet.launches_per_step counts the optimiser's launches as the library makes them."""
    from paper_2607_14672_gb300 import net

    class Sized:
        def __init__(self, n):
            self.numel = lambda: n

    stub = net.Clipped()
    stub.W, stub.max_norm = [Sized(n) for n in sizes], 0.5
    code, made = step(lib, list(sizes))
    assert code == OK and stub.optimizer_launches() == len(made)
    stub.max_norm = None
    assert stub.optimizer_launches() == 1


def plan(lib, T, N, K):
    """Width, form of the work and whether the sides are exchanged, from the tensor-core launch's own argument:
    T, N, K, two truth values (weights copied, sides exchanged), then the plan's width, tiles along N and T,
    blocks of K, whole tiles, and blocks of a share of the others."""
    lib.fake_keep_arg2_of(b"k_q8_tc")
    assert product(lib, T, N, K, ld=row_stride(K)) == OK
    name, grid, _, _ = fake_cuda.launches(lib)[-1]
    assert "k_q8_tc" in name
    a = bytes(lib.fake_arg2(lib.fake_launches() - 1).contents)
    t, n, k, copied, exchanged, nt, tiles_n, tiles_t, blocks, whole, share = struct.unpack("3i2?2x6i", a[:40])
    assert (t, n, k) == ((N, T, K) if exchanged else (T, N, K)) and not copied
    assert f"ILi{nt}E" in name
    tiles = tiles_n * tiles_t
    assert tiles == -(-n // 256) * -(-t // nt) and blocks == -(-k // 128) and 0 <= whole <= tiles
    assert (share > 0) == (whole < tiles)
    if share:
        assert share * (grid // 2) >= (tiles - whole) * blocks     # the shares cover what is cut
    return nt, "one piece" if not share else ("whole and cut" if whole else "cut"), exchanged


@pytest.mark.parametrize("T,N,K,nt,form,exchanged", PLANS)
def test_plans_of_the_tested_shapes(lib, T, N, K, nt, form, exchanged):
    """The shapes whose results are compared on the GPU reach what they are there for."""
    assert plan(lib, T, N, K) == (nt, form, exchanged)


def test_every_width_is_tested_in_every_form():
    assert {p[3:] for p in PLANS} == {(nt, form, exchanged) for nt in (32, 64, 96, 128, 160, 192)
                                      for form in ("one piece", "cut", "whole and cut") for exchanged in (False, True)}


@pytest.mark.parametrize("B,N_in,N_out,M,writers,tc,exchanged", [
    (2, 5000, 60, 16, 2, True, False), (2, 9001, 40, 32, 3, True, True), (2, 16384, 50, 8, 4, True, False),
    (64, 300, 21, 32, 1, True, True), (128, 2000, 40, 32, 1, False, None), (64, 1500, 130, 32, 1, True, True)])
def test_launches_of_the_tested_layers(lib, B, N_in, N_out, M, writers, tc, exchanged):
    """The layers whose spike times are compared on the GPU reach several blocks a sample of the token writer, both
    forms of the product, and either side first."""
    from paper_2607_14672_gb300 import dstd
    p = dstd.params(dict(tau_v=0.5, tau_I=0.25, v_th=1.0, t_first=0.0, t_end=1.2, M=M, t_offset=0.0), 1.0 / B)
    lib.fake_keep_arg2_of(b"k_q8_tc")
    need = lib.dstd_dense_q8_workspace_bytes(B, N_in, N_out, ctypes.byref(p))
    assert lib.dstd_dense_fwd_q8(P, P, P, B, N_in, N_out, ctypes.byref(p), P, P, None, P, need, None) == OK
    names = fake_cuda.launches(lib)
    assert "k_bin_codes" in names[0][0] and names[0][1] == writers
    where = [i for i, n in enumerate(names) if "k_q8_tc" in n[0]]
    assert bool(where) == tc
    if tc:
        assert struct.unpack("2?", bytes(lib.fake_arg2(where[0]).contents)[12:14])[1] == exchanged

"""Host code of the 4-bit and distillation calls, without a GPU: what is launched, and the set-up on each device
(through a runtime that runs nothing, see fake_cuda.cpp)."""

import ctypes
import struct

import pytest

import fake_cuda
from mx4_plans import PLANS

pytestmark = pytest.mark.skipif(fake_cuda.compiler() is None, reason="no C++ compiler")

P = ctypes.c_void_p(256)
OK = 0
F = ctypes.c_float


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


def product(lib, T, N, K, out_type=0):
    row = (K + 31) // 32 * 16
    return lib.dstd_mx4_matmul(P, row, P, P, row, P, T, N, K, P, out_type, N, None)


@pytest.mark.parametrize("out_type", [0, 1, 2])
@pytest.mark.parametrize("T,N,K,width,parts,exchanged", PLANS)
def test_plans(lib, T, N, K, width, parts, exchanged, out_type):
    lib.fake_keep_arg2_of(b"k_mx4_tc")
    assert product(lib, T, N, K, out_type) == OK
    (name, grid, block, _), = fake_cuda.launches(lib)
    if width == 0:
        assert "k_mx4_pair" in name and grid <= 152 and grid % 2 == 0 and block == 320
        return
    assert f"k_mx4_tcILi{width}E" in name and block == 192
    a, rows_a, _, b, rows_b, _, blocks, ktiles, tiles_a, tiles_b, got, slots = struct.unpack(
        "<QiiQiiiiiiii", bytes(lib.fake_arg2(0).contents)[:56])
    assert (rows_a, rows_b) == ((T, N) if exchanged else (N, T)) and got == parts
    assert blocks == -(-K // 32) and ktiles == -(-blocks // 4)
    assert tiles_a == -(-rows_a // 128) and tiles_b == -(-rows_b // width) and grid == tiles_a * tiles_b * parts
    assert tiles_b == 1 or width == 128                 # scales are in tiles of 128 rows
    assert parts <= -(-blocks // 8) and slots >= 3


@pytest.mark.parametrize("T", [1, 16, 17, 40, 100, 1000])
@pytest.mark.parametrize("N", [1, 128, 500, 2500, 20000])
def test_no_part_without_columns(lib, T, N):
    """A block whose share of K is empty would wait for sums that nobody forms; blocks that share K have an SM each."""
    for K in (1, 32, 33, 256, 257, 512, 513, 1000, 1025, 2000, 2049, 5000, 40000):
        lib.fake_reset()
        lib.fake_keep_arg2_of(b"k_mx4_tc")
        assert product(lib, T, N, K) == OK
        (name, grid, _, _), = fake_cuda.launches(lib)
        if "k_mx4_pair" in name:
            continue
        parts = struct.unpack("<QiiQiiiiiiii", bytes(lib.fake_arg2(0).contents)[:56])[10]
        assert 1 <= parts <= -(-K // 256) and (parts == 1 or grid <= 152), (K, parts, grid)


def test_the_plans_reach_every_form():
    assert {(w, p) for _, _, _, w, p, _ in PLANS} >= {(16, 1), (16, 2), (16, 4), (16, 8), (32, 1), (64, 1), (64, 2), (64, 4),
                                                      (64, 8), (128, 1), (128, 2), (128, 4), (128, 8), (0, 1)}
    assert {w for _, _, _, w, _, e in PLANS if e} >= {16, 32, 64}


@pytest.mark.parametrize("T,N", [(2 ** 31 - 2048, 1), (1, 2 ** 31 - 2048), (2 ** 31 - 2048, 128)])
def test_the_largest_sizes_are_taken(lib, T, N):
    assert product(lib, T, N, 32) == OK
    (name, grid, _, _), = fake_cuda.launches(lib)
    assert 0 < grid <= 2 ** 24


def test_nothing_to_do(lib):
    assert product(lib, 0, 5, 32) == OK and product(lib, 5, 0, 32) == OK and lib.fake_launches() == 0
    assert product(lib, 5, 7, 0) == OK
    assert "k_zero_rows" in fake_cuda.launches(lib)[0][0]
    assert lib.dstd_quantize_mx4(P, 0, 0, 40, 40, P, 32, P, None, 0, None) == OK
    assert lib.dstd_quantize_mx4(P, 0, 4, 0, 0, P, 0, P, None, 0, None) == OK
    assert lib.fake_launches() == 1


def distill(lib, R, C, K, type=0, silent=float("-inf")):
    return lib.dstd_distill_loss(P, type, R, C, C, F(1.0), F(silent), P, P, K, F(1.0), F(1.0), None, P, P, ctypes.c_void_p(1 << 20), C, 0, None)


def top(lib, R, C, K, type=0):
    return lib.dstd_top_logits(P, type, R, C, C, F(1.0), F(float("-inf")), K, P, P, None)


CALLS = {
    "product of blocks": lambda lib: product(lib, 8, 4096, 4096),
    "product of pairs": lambda lib: product(lib, 4096, 4096, 4096),
    "largest logits": lambda lib: top(lib, 3, 100000, 64),
    "distillation": lambda lib: distill(lib, 3, 100000, 64),
}


@pytest.mark.parametrize("what", CALLS)
def test_on_another_device(loaded, what):
    """The grant of shared memory, and the pairs that fit, belong to a device."""
    lib = fake_cuda.load()                            # a library that has launched nothing yet
    lib.fake_reset()
    for device in (0, 1, 2, 0):
        lib.fake_device(device)
        before = lib.fake_launches()
        assert CALLS[what](lib) == OK
        (name, grid, _, at), = fake_cuda.launches(lib)[before:]
        assert at == device
        if what == "product of pairs":
            assert grid == 2 * (50 if device == 2 else 76)


@pytest.mark.parametrize("what", [what for what in CALLS if what not in ("largest logits", "distillation")])   # which ask for none
def test_after_a_failure(loaded, what):
    """A runtime call that fails once fails that call, and no later one."""
    lib = fake_cuda.load()
    lib.fake_reset()
    lib.fake_refuse_attributes(1)
    assert CALLS[what](lib) != OK
    assert CALLS[what](lib) == OK


def test_rows_are_shared_only_where_they_are_few(lib):
    for R, C, parts in [(1, 131072, 8), (7, 131071, 8), (40, 131072, 4), (200, 131072, 1), (4096, 32768, 1), (3, 5000, 2), (3, 3000, 1)]:
        for call in (distill, top):
            before = lib.fake_launches()
            assert call(lib, R, C, 100) == OK
            (name, grid, _, _), *rest = fake_cuda.launches(lib)[before:]
            assert grid == R * parts, (name, R, C, grid)
            assert [n for n, *_ in rest] == [] if call is top or R <= 304 else "k_distill_sum" in rest[0][0] and len(rest) == 1


def test_short_rows_take_a_warp(lib):
    for R, C, K, type, name in [(256, 10, 4, 0, "k_distill_small"), (9, 64, 64, 1, "k_distill_small"), (9, 65, 64, 0, "k_distill_packsIfLi2E"),
                                (17, 256, 64, 0, "k_distill_packsIfLi2E"), (17, 257, 64, 0, "k_distill_packsIfLi8E"),
                                (17, 512, 64, 2, "k_distill_packsI6__halfLi2E"), (17, 2048, 64, 2, "k_distill_packsI6__halfLi8E"),
                                (17, 1024, 64, 0, "k_distill_packsIfLi8E"), (17, 1025, 64, 0, "k_distillI"), (17, 2049, 64, 1, "k_distillI"),
                                (17, 10, 65, 0, "k_distillI"), (608, 1000, 65, 0, "k_distillI"), (609, 1000, 65, 0, "k_distill_packsIfLi8ELi4E"),
                                (609, 2048, 128, 2, "k_distill_packsI6__halfLi8ELi4E"), (609, 1000, 129, 0, "k_distillI"), (609, 1025, 65, 0, "k_distillI")]:
        before = lib.fake_launches()
        assert distill(lib, R, C, K, type) == OK
        got, grid, _, _ = fake_cuda.launches(lib)[before]
        assert name in got and grid == (R if name == "k_distillI" else -(-R // 8))
    for R, C, K, type, name in [(256, 10, 4, 0, "k_top_small"), (9, 33, 5, 0, "k_top_packsIfLi8E"), (9, 256, 64, 1, "k_top_packsI13__nv_bfloat16Li8E"),
                                (9, 257, 64, 0, "k_top_logits"), (760, 257, 64, 0, "k_top_logits"), (761, 257, 64, 0, "k_top_packsIfLi16E"),
                                (761, 513, 64, 0, "k_top_packsIfLi32E"), (761, 1024, 64, 2, "k_top_packsI6__halfLi32E"), (761, 1025, 5, 0, "k_top_logits"),
                                (9, 128, 65, 0, "k_top_small"), (9, 129, 65, 0, "k_top_logits"),
                                (761, 129, 65, 0, "k_top_packsIfLi8E"), (761, 1024, 128, 0, "k_top_packsIfLi32E"), (761, 1024, 129, 0, "k_top_logits")]:
        before = lib.fake_launches()
        assert top(lib, R, C, K, type) == OK
        (got, grid, _, _), = fake_cuda.launches(lib)[before:]
        assert name in got and grid == (R if name == "k_top_logits" else -(-R // 8))

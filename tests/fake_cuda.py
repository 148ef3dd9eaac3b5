"""The library's host code on a machine without a GPU: its objects linked against
a CUDA runtime that runs nothing and writes down every launch (fake_cuda.cpp)."""

import ctypes
import os
import shutil
import subprocess
import tempfile

HERE = os.path.dirname(os.path.abspath(__file__))


def compiler():
    return shutil.which("g++") or shutil.which("c++")


def load():
    """The library with the fake runtime; its entry points take the addresses and sizes that the real ones do."""
    from paper_2607_14672_gb300 import build, dstd
    build.build()
    cuda = os.path.dirname(os.path.dirname(os.path.realpath(build.nvcc_path())))
    objects = [os.path.join(build.BUILD_DIR, os.path.splitext(s)[0] + ".o") for s in build.SOURCES]
    folder = tempfile.mkdtemp(prefix="dstd_fake_")
    try:
        path = os.path.join(folder, "libdstd_fake.so")
        # -Bsymbolic: its own runtime calls, whatever else the process has loaded
        subprocess.run([compiler(), "-std=c++17", "-O1", "-fPIC", "-shared", "-I", os.path.join(cuda, "include"),
                        "-Wl,-Bsymbolic", "-Wl,--no-undefined", "-o", path, os.path.join(HERE, "fake_cuda.cpp")] +
                       objects + ["-lpthread"], check=True, capture_output=True)
        lib = ctypes.CDLL(path)
    finally:
        shutil.rmtree(folder)
    for name in dstd.EXPORTS:
        mine, real = getattr(lib, name), getattr(dstd.load(), name)
        mine.restype, mine.argtypes = real.restype, real.argtypes
    lib.fake_name.restype = ctypes.c_char_p
    lib.fake_arg2.restype = ctypes.POINTER(ctypes.c_ubyte * 64)
    lib.fake_keep_arg2_of.argtypes = [ctypes.c_char_p]
    lib.fake_grid.restype = lib.fake_block.restype = ctypes.c_uint
    return lib


def launches(lib):
    """(kernel's name, grid, block, device) of each launch since the last reset."""
    return [(lib.fake_name(i).decode(), lib.fake_grid(i), lib.fake_block(i), lib.fake_launch_device(i))
            for i in range(lib.fake_launches())]

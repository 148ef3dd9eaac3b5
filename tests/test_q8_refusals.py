"""CPU checks of the 8-bit and clipping entry points: argument checks on the
host, before anything is launched (no GPU needed)."""

import ctypes
import math
import os
import shutil

import pytest
import torch

pytestmark = pytest.mark.skipif(shutil.which("nvcc") is None and not os.path.exists("/usr/local/cuda/bin/nvcc"),
                                reason="nvcc not available")

P = ctypes.c_void_p(256)
ODD = ctypes.c_void_p(258)
INVALID, UNSUPPORTED, WORKSPACE = -1, -2, -3


@pytest.fixture(scope="module")
def lib():
    from paper_2607_14672_gb300 import build, dstd
    build.build()
    return dstd.load()


def layer(M=32):
    from paper_2607_14672_gb300 import dstd
    return dstd.params(dict(tau_v=0.5, tau_I=0.25, v_th=1.0, t_first=0.0, t_end=1.2, M=M, t_offset=0.0), 1.0 / 8)


@pytest.mark.parametrize("args", [
    (None, 0, 4, 8, 8, P, 8, P, None, 0),    # no x
    (P, 3, 4, 8, 8, P, 8, P, None, 0),       # unknown type
    (P, 0, -1, 8, 8, P, 8, P, None, 0),      # negative rows
    (P, 0, 4, -8, 8, P, 8, P, None, 0),      # negative columns
    (P, 0, 4, 8, 7, P, 8, P, None, 0),       # overlapping rows of x
    (P, 0, 4, 8, 8, P, 7, P, None, 0),       # overlapping rows of q
    (P, 0, 4, 8, 8, None, 8, P, None, 0),    # no q
    (P, 0, 4, 8, 8, P, 8, None, None, 0),    # no scale
    (P, 0, 4, 8, 8, P, 8, P, P, 7),          # overlapping rows of values
    (ODD, 0, 4, 8, 8, P, 8, P, None, 0),     # fp32 at half an element
    (P, 0, 4, 8, 8, P, 8, ODD, None, 0),
])
def test_quantize_rows_refuses(lib, args):
    assert lib.dstd_quantize_rows(*args, None) == INVALID


def test_int8_matmul_refuses(lib):
    ok = dict(x=P, ld_x=16, xs=P, w=P, ld_w=16, ws=P, T=4, N=8, K=16, out=P, type=0, ld_out=8, wsp=P,
              bytes=1 << 30)

    def call(**kw):
        return lib.dstd_int8_matmul(*dict(ok, **kw).values(), None)

    for bad in (dict(x=None), dict(w=None), dict(xs=None), dict(ws=None), dict(out=None), dict(wsp=None),
                dict(T=-1), dict(N=-1), dict(K=-1), dict(ld_x=15), dict(ld_w=15), dict(ld_out=7), dict(type=5),
                dict(out=ODD), dict(xs=ODD), dict(ws=ODD), dict(wsp=ODD)):
        assert call(**bad) == INVALID, bad
    assert call(K=131072, ld_x=131072, ld_w=131072) == UNSUPPORTED
    assert call(bytes=0) == WORKSPACE
    assert lib.dstd_int8_matmul_workspace_bytes(4, 8, 16) > 0
    for bad in ((-1, 8, 16), (4, -8, 16), (4, 8, -16), (4, 8, 131072)):
        assert lib.dstd_int8_matmul_workspace_bytes(*bad) == 0, bad
        assert lib.dstd_int8_matmul_aligned_workspace_bytes(*bad) == 0, bad
    # the weights' copy is what the aligned size leaves out
    full, small = (f(64, 1000, 2048) for f in (lib.dstd_int8_matmul_workspace_bytes,
                                               lib.dstd_int8_matmul_aligned_workspace_bytes))
    assert abs((full - small) - 1000 * 2048) <= 256


def test_dense_fwd_q8_refuses(lib):
    p = ctypes.byref(layer())
    ok = dict(t=P, wq=P, ws=P, B=8, N_in=16, N_out=16, p=p, t_out=P, saved=P, pen=None, wsp=P, bytes=1 << 30)

    def call(**kw):
        return lib.dstd_dense_fwd_q8(*dict(ok, **kw).values(), None)

    for bad in (dict(t=None), dict(wq=None), dict(ws=None), dict(t_out=None), dict(saved=None), dict(wsp=None),
                dict(p=None), dict(B=0), dict(N_in=0), dict(N_out=0), dict(wq=ODD)):
        assert call(**bad) == INVALID, bad
    assert call(bytes=16) == WORKSPACE
    long = layer(M=200)
    assert call(p=ctypes.byref(long)) == UNSUPPORTED
    assert call(N_in=131072) == UNSUPPORTED
    from paper_2607_14672_gb300 import dstd
    assert dstd.dense_q8_workspace_bytes(8, 16, 16, layer()) > 0
    assert dstd.dense_q8_workspace_bytes(8, 16, 16, long) == 0
    assert dstd.dense_q8_workspace_bytes(0, 16, 16, layer()) == 0


def lists(n=(10, 3), ptr=256, type=0):
    k = len(n)
    return ((ctypes.c_void_p * k)(*[ptr] * k), (ctypes.c_int64 * k)(*n), (ctypes.c_int32 * k)(*[type] * k))


def test_tensor_lists_refused(lib):
    g, n, ty = lists()

    def norm(count=2, g=g, n=n, ty=ty, norm=P, wsp=P, bytes=1 << 30):
        return lib.dstd_grad_norm(count, g, n, ty, norm, None, wsp, bytes, None)

    assert norm(count=0) == INVALID
    assert norm(g=None) == INVALID and norm(n=None) == INVALID and norm(ty=None) == INVALID
    assert norm(norm=None) == INVALID and norm(wsp=None) == INVALID and norm(wsp=ODD) == INVALID
    assert norm(n=lists((10, -1))[1]) == INVALID
    assert norm(ty=lists(type=3)[2]) == INVALID
    assert norm(g=lists(ptr=0)[0]) == INVALID
    assert norm(g=lists(ptr=258)[0]) == INVALID       # fp32 at half an element
    assert norm(n=lists((10, 1 << 60))[1]) == UNSUPPORTED
    assert norm(bytes=16) == WORKSPACE
    assert lib.dstd_grad_norm_workspace_bytes(2, n) > 0
    assert lib.dstd_grad_norm_workspace_bytes(0, n) == 0
    assert lib.dstd_grad_norm_workspace_bytes(2, None) == 0
    assert lib.dstd_grad_norm_workspace_bytes(2, lists((10, -1))[1]) == 0
    assert lib.dstd_grad_norm_workspace_bytes(2, lists((1 << 60, 1 << 60))[1]) == 0


def test_clip_and_step_refused(lib):
    g, n, ty = lists()

    def clip(max_norm=1.0, out=g):
        return lib.dstd_clip_grads(2, g, out, n, ty, max_norm, P, P, 1 << 30, None)

    for bad in (0.0, -1.0, math.nan):
        assert clip(max_norm=bad) == INVALID
    assert clip(out=None) == INVALID and clip(out=lists(ptr=0)[0]) == INVALID

    def step(w=g, m=g, v=g, lr=1e-3, b1=0.9, b2=0.999, eps=1e-8, wd=1e-2, max_norm=1.0, step=P):
        return lib.dstd_adamw_clip(2, w, g, m, v, n, ty, lr, b1, b2, eps, wd, max_norm, step, None, P, P, 1 << 30,
                                   None)

    for bad in (dict(w=None), dict(m=None), dict(v=None), dict(step=None), dict(step=ODD), dict(w=lists(ptr=0)[0]),
                dict(m=lists(ptr=258)[0]), dict(lr=-1.0), dict(lr=math.nan), dict(b1=1.0), dict(b1=-0.1),
                dict(b2=1.0), dict(eps=0.0), dict(eps=1e-60), dict(wd=math.inf), dict(max_norm=0.0)):
        assert step(**bad) == INVALID, bad


def test_binding_checks_tensors(lib):
    """The binding refuses what is not on the GPU, before any pointer is taken."""
    from paper_2607_14672_gb300 import dstd
    x = torch.zeros(4, 8)
    with pytest.raises(ValueError):
        dstd.quantize_rows(x, torch.zeros(4, 8, dtype=torch.int8), torch.zeros(4))
    with pytest.raises(ValueError):
        dstd.int8_matmul(x.to(torch.int8), torch.zeros(4), x.to(torch.int8), torch.zeros(4), torch.zeros(4, 4), x)
    with pytest.raises(ValueError):
        dstd.TensorList([x])

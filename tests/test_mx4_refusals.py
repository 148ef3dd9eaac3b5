"""CPU checks of the 4-bit and distillation entry points: argument checks on the
host, before anything is launched, and the binding's checks (no GPU needed)."""

import ctypes
import math
import shutil
import os

import pytest
import torch

from test_binding_devices import codes, floats, made, p, put  # noqa: F401  (made is a fixture)

pytestmark = pytest.mark.skipif(shutil.which("nvcc") is None and not os.path.exists("/usr/local/cuda/bin/nvcc"),
                                reason="nvcc not available")

P, ODD, OFF = ctypes.c_void_p(256), ctypes.c_void_p(258), ctypes.c_void_p(257)
HALF = ctypes.c_void_p(264)                       # a multiple of 8, not of 16
INVALID, UNSUPPORTED, WORKSPACE = -1, -2, -3
TOP = 2 ** 31 - 1


@pytest.fixture(scope="module")
def lib():
    from paper_2607_14672_gb300 import build, dstd
    build.build()
    return dstd.load()


def test_sizes(lib):
    f = lib.dstd_mx4_scale_bytes
    assert f(-1, 5) == 0 and f(5, -1) == 0 and f(0, 5) == 0 and f(5, 0) == 0
    assert f(1, 1) == 512 and f(128, 128) == 512 and f(129, 129) == 2048
    assert f(TOP, TOP) == 2 ** 24 * 2 ** 24 * 512
    from paper_2607_14672_gb300 import dstd
    assert [dstd.mx4_row_bytes(k) for k in (0, 1, 32, 33, 16384)] == [0, 16, 16, 32, 8192]
    for r, c in ((0, 5), (5, 0), (1, 1), (128, 128), (129, 129), (800, 784), (16384, 16385)):
        assert dstd.mx4_scale_bytes(r, c) == f(r, c)


QUANT = dict(x=P, type=0, rows=4, cols=40, ld_x=40, q=P, ld_q=32, scale=P, values=P, ld_v=40)


@pytest.mark.parametrize("bad", [dict(x=None), dict(type=3), dict(type=-1), dict(rows=-1), dict(cols=-1), dict(ld_x=39),
                                 dict(q=None), dict(q=HALF), dict(ld_q=16), dict(ld_q=40), dict(ld_q=-32),
                                 dict(scale=None), dict(scale=HALF), dict(values=ODD), dict(ld_v=39), dict(x=ODD)])
def test_quantize_refuses(lib, bad):
    assert lib.dstd_quantize_mx4(*dict(QUANT, **bad).values(), None) == INVALID


def test_quantize_sizes(lib):
    big = dict(rows=1, cols=TOP - 2047 + 1, ld_x=TOP, ld_q=2 ** 31, ld_v=TOP)
    assert lib.dstd_quantize_mx4(*dict(QUANT, **big).values(), None) == UNSUPPORTED


MATMUL = dict(x=P, ld_x=32, xs=P, w=P, ld_w=32, ws=P, T=4, N=8, K=40, out=P, type=0, ld_out=8)


@pytest.mark.parametrize("bad", [dict(x=None), dict(w=None), dict(xs=None), dict(ws=None), dict(out=None), dict(x=HALF),
                                 dict(w=HALF), dict(xs=HALF), dict(ws=HALF), dict(ld_x=16), dict(ld_w=40), dict(T=-1),
                                 dict(N=-1), dict(K=-1), dict(type=4), dict(out=ODD), dict(ld_out=7)])
def test_matmul_refuses(lib, bad):
    assert lib.dstd_mx4_matmul(*dict(MATMUL, **bad).values(), None) == INVALID


@pytest.mark.parametrize("big", [dict(T=TOP - 2046), dict(N=TOP - 2046, ld_out=TOP), dict(K=TOP - 2046, ld_x=2 ** 31, ld_w=2 ** 31)])
def test_matmul_sizes(lib, big):
    assert lib.dstd_mx4_matmul(*dict(MATMUL, **big).values(), None) == UNSUPPORTED


def test_layer_refuses(lib):
    pp = ctypes.byref(p)
    ok = dict(t=P, w=P, ws=P, B=4, n_in=40, n_out=8, p=pp, t_out=P, saved=P, pen=P, wsp=P, bytes=1 << 30)
    call = lambda **kw: lib.dstd_dense_fwd_mx4(*dict(ok, **kw).values(), None)
    for bad in (dict(t=None), dict(w=None), dict(ws=None), dict(t_out=None), dict(saved=None), dict(wsp=None), dict(B=0),
                dict(n_in=0), dict(n_out=0), dict(p=None), dict(t=HALF), dict(w=HALF), dict(ws=HALF), dict(wsp=HALF),
                dict(saved=HALF)):
        assert call(**bad) == INVALID, bad
    assert call(bytes=64) == WORKSPACE
    from paper_2607_14672_gb300 import dstd
    wide = dstd.params(dict(tau_v=0.5, tau_I=0.25, v_th=1.0, t_first=0.0, t_end=1.2, M=200, t_offset=0.0), 1.0)
    assert call(p=ctypes.byref(wide)) == UNSUPPORTED
    assert dstd.dense_mx4_workspace_bytes(4, 40, 8, wide) == 0
    assert dstd.dense_mx4_workspace_bytes(0, 40, 8, p) == 0
    need = dstd.dense_mx4_workspace_bytes(4, 40, 8, p)
    assert need >= 4 * 8 * (32 + 8 * 4) and call(bytes=need - 1) == WORKSPACE


F = ctypes.c_float
TOPK = dict(y=P, type=0, R=4, C=10, ld=10, factor=F(1.0), silent=F(-math.inf), K=3, top=P, index=P)
LOSS = dict(y=P, type=0, R=4, C=10, ld=10, factor=F(1.0), silent=F(-math.inf), top=P, index=P, K=3, tf=F(1.0),
            weight=F(1.0), rw=P, loss=P, rows=P, g=ctypes.c_void_p(1 << 20), ld_g=10, acc=0)
COMMON = [dict(y=None), dict(type=3), dict(R=0), dict(C=0), dict(ld=9), dict(y=ODD), dict(factor=F(0.0)),
          dict(factor=F(math.inf)), dict(factor=F(math.nan)), dict(silent=F(math.inf)), dict(silent=F(math.nan)),
          dict(factor=F(-1.0)), dict(K=0), dict(top=None), dict(index=None), dict(top=ODD), dict(index=ODD)]


@pytest.mark.parametrize("bad", COMMON + [dict(K=11)])
def test_top_refuses(lib, bad):
    assert lib.dstd_top_logits(*dict(TOPK, **bad).values(), None) == INVALID


@pytest.mark.parametrize("bad", COMMON + [dict(rw=ODD), dict(loss=None), dict(loss=ctypes.c_void_p(260)), dict(rows=None),
                                          dict(rows=ODD), dict(g=ODD), dict(g=P), dict(ld_g=9), dict(tf=F(0.0)), dict(tf=F(math.nan)),
                                          dict(weight=F(math.inf))])
def test_loss_refuses(lib, bad):
    assert lib.dstd_distill_loss(*dict(LOSS, **bad).values(), None) == INVALID


def test_long_records_and_rows(lib):
    wide = dict(C=2 ** 30 + 1, ld=2 ** 30 + 1)
    assert lib.dstd_top_logits(*dict(TOPK, **wide).values(), None) == UNSUPPORTED
    assert lib.dstd_distill_loss(*dict(LOSS, **wide, ld_g=2 ** 31).values(), None) == UNSUPPORTED
    assert lib.dstd_top_logits(*dict(TOPK, C=1000, ld=1000, K=257).values(), None) == UNSUPPORTED
    assert lib.dstd_distill_loss(*dict(LOSS, K=257).values(), None) == UNSUPPORTED


# -- the binding -----------------------------------------------------------
def u8(*shape):
    return torch.zeros(*shape, dtype=torch.uint8)


def i32(*shape):
    return torch.zeros(*shape, dtype=torch.int32)


def aligned(x):
    """A copy at a multiple of 16 bytes."""
    store = torch.zeros(x.numel() + 16, dtype=x.dtype)
    at = (-store.data_ptr() % 16) // x.element_size()
    return store[at:at + x.numel()].view(x.shape)


def calls():
    from paper_2607_14672_gb300 import dstd
    return {
        "quantize_mx4": (lambda t, **k: dstd.quantize_mx4(*t, **k), [floats(4, 40), u8(4, 32), u8(512), floats(4, 40)]),
        "mx4_matmul": (lambda t, **k: dstd.mx4_matmul(*t, **k), [u8(4, 32), u8(512), u8(5, 32), u8(512), floats(4, 5)]),
        "dense_fwd_mx4": (lambda t, **k: dstd.dense_fwd_mx4(t[0], t[1], t[2], p, t[3], None, None, t[4], **k),
                          [floats(4, 40), u8(5, 32), u8(512), floats(4, 5), u8(64)]),
        "top_logits": (lambda t, **k: dstd.top_logits(*t, **k), [floats(4, 9), floats(4, 3), i32(4, 3)]),
        "distill_loss": (lambda t, **k: dstd.distill_loss(*t[:6], row_weight=t[6], **k),
                         [floats(4, 9), floats(4, 3), i32(4, 3), floats(2), floats(4), floats(4, 9), floats(4)]),
    }


@pytest.mark.parametrize("stream", [None, 7])
@pytest.mark.parametrize("name", ["quantize_mx4", "mx4_matmul", "dense_fwd_mx4", "top_logits", "distill_loss"])
def test_tensors_of_another_device_are_refused(made, name, stream):  # noqa: F811
    call, tensors = calls()[name]
    call([put(aligned(x), 0) for x in tensors], stream=stream)
    assert made == ["dstd_" + name]
    with pytest.raises(ValueError):
        call([put(aligned(x), 1) for x in tensors], stream=stream)
    for other in range(len(tensors)):
        with pytest.raises(ValueError):
            call([put(aligned(x), int(i == other)) for i, x in enumerate(tensors)], stream=stream)
    assert made == ["dstd_" + name]


@pytest.mark.parametrize("name,at,bad", [
    ("quantize_mx4", 0, floats(4, 40).double()), ("quantize_mx4", 0, floats(40, 4).t()), ("quantize_mx4", 1, u8(4, 16)),
    ("quantize_mx4", 1, u8(5, 32)), ("quantize_mx4", 1, codes(4, 32)), ("quantize_mx4", 1, u8(4, 40)[:, :32]),
    ("quantize_mx4", 1, u8(4 * 32 + 8)[8:].view(4, 32)), ("quantize_mx4", 2, u8(511)), ("quantize_mx4", 2, codes(512)),
    ("quantize_mx4", 3, floats(4, 39)), ("quantize_mx4", 3, floats(4, 40).half()),
    ("mx4_matmul", 0, u8(4, 24)), ("mx4_matmul", 2, u8(5, 48)), ("mx4_matmul", 1, u8(100)), ("mx4_matmul", 3, u8(1024)[::2]),
    ("mx4_matmul", 4, floats(5, 4)), ("mx4_matmul", 4, floats(4, 5).double()), ("mx4_matmul", 4, floats(5, 4).t()),
    ("dense_fwd_mx4", 1, u8(5, 48)), ("dense_fwd_mx4", 1, u8(5, 64)[:, :32]), ("dense_fwd_mx4", 2, u8(100)),
    ("dense_fwd_mx4", 3, floats(4, 6)),
    ("top_logits", 0, floats(4, 9).double()), ("top_logits", 0, floats(9, 4).t()), ("top_logits", 1, floats(3, 3)),
    ("top_logits", 1, floats(4, 3).half()), ("top_logits", 2, i32(4, 2)), ("top_logits", 2, i32(4, 3).long()),
    ("top_logits", 2, i32(4, 6)[:, ::2]),
    ("distill_loss", 1, floats(4, 6)[:, ::2]), ("distill_loss", 2, i32(4, 3).long()), ("distill_loss", 3, floats(1)),
    ("distill_loss", 4, floats(5)), ("distill_loss", 5, floats(4, 9).half()), ("distill_loss", 5, floats(4, 8)),
    ("distill_loss", 6, floats(3))])
def test_shapes_and_types_are_refused(made, name, at, bad):  # noqa: F811
    call, tensors = calls()[name]
    tensors = [put(aligned(x), 0) for x in tensors]
    tensors[at] = put(bad, 0)
    with pytest.raises(ValueError):
        call(tensors)
    assert made == []

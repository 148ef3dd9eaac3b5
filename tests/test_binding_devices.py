"""The binding's checks of devices, without a GPU: kernels run on the current
device, and a tensor of another one would be out of their reach. Tensors here
are host tensors that say they are on a device."""

import pytest
import torch

from paper_2607_14672_gb300 import dstd


class OnDevice(torch.Tensor):
    index = 0
    is_cuda = True

    def get_device(self):
        return self.index


def put(x, index):
    x = x.as_subclass(OnDevice)
    x.index = index
    return x


@pytest.fixture
def made(monkeypatch):
    """The calls that reach the library, which is not there; device 0 is the current one."""
    calls = []

    class Library:
        def __getattr__(self, name):
            return lambda *a: calls.append(name) or 0
    dstd._torch()
    monkeypatch.setattr(dstd, "_DEVICE", lambda: 0, raising=False)
    monkeypatch.setattr(dstd, "_ONLY", -2, raising=False)
    monkeypatch.setattr(dstd, "_RAW_STREAM", lambda index: 1000 + index)
    monkeypatch.setattr(dstd, "load", lambda: Library())
    return calls


def floats(*shape):
    return torch.zeros(*shape)


def codes(*shape):
    return torch.zeros(*shape, dtype=torch.int8)


p = dstd.params(dict(tau_v=0.5, tau_I=0.25, v_th=1.0, t_first=0.0, t_end=1.2, M=8, t_offset=0.0), 1.0)
CALLS = {
    "quantize_rows": (lambda t, **k: dstd.quantize_rows(*t, **k), [floats(4, 8), codes(4, 8), floats(4), floats(4, 8)]),
    "int8_matmul": (lambda t, **k: dstd.int8_matmul(*t, **k),
                    [codes(4, 8), floats(4), codes(5, 8), floats(5), floats(4, 5), codes(64)]),
    "dense_fwd_q8": (lambda t, **k: dstd.dense_fwd_q8(t[0], t[1], t[2], p, t[3], None, None, t[4], **k),
                     [floats(4, 8), codes(5, 8), floats(5), floats(4, 5), codes(64)]),
    "grad_norm": (lambda t, **k: dstd.grad_norm([t[0]], t[1], t[2], t[3], **k),
                  [floats(9), floats(1), codes(64), floats(1)]),
    "clip_grads": (lambda t, **k: dstd.clip_grads([t[0]], 1.0, t[1], t[2], [t[3]], **k),
                   [floats(9), floats(1), codes(64), floats(9)]),
    "adamw_clip": (lambda t, **k: dstd.adamw_clip([t[0]], [t[1]], [t[2]], [t[3]], 1e-3, 0.9, 0.999, 1e-8, 0.0, t[4], 1.0,
                                                  t[5], t[6], lr_dev=t[7], **k),
                   [floats(9), floats(9), floats(9), floats(9), torch.zeros(1, dtype=torch.int32), floats(1), codes(64),
                    floats(1)]),
}


@pytest.mark.parametrize("stream", [None, 7])
@pytest.mark.parametrize("name", CALLS)
def test_tensors_of_another_device_are_refused(made, name, stream):
    call, tensors = CALLS[name]
    call([put(x.clone(), 0) for x in tensors], stream=stream)
    assert made == ["dstd_" + name]
    with pytest.raises(ValueError):          # all of them on a device that is not the current one
        call([put(x.clone(), 1) for x in tensors], stream=stream)
    for other in range(len(tensors)):        # one of them
        with pytest.raises(ValueError):
            call([put(x.clone(), int(i == other)) for i, x in enumerate(tensors)], stream=stream)
    assert made == ["dstd_" + name]


def test_lists_of_two_devices_are_refused():
    with pytest.raises(ValueError):
        dstd.TensorList([put(floats(3), 0), put(floats(3), 1)])

"""Clipped steps of the networks, and gradients at the ends of the ranges, on the
GPU. Tolerances as derived in the tests of ordinary lists: NORM for the norm,
FACTOR for the clip factor."""

import math

import pytest
import torch

from test_gpu_clip import FACTOR, NORM, U, host, lib, norms, workspace  # noqa: F401 (lib is a fixture)

pytestmark = pytest.mark.gpu


def small_conv(max_norm):
    from paper_2607_14672_gb300 import configs, net
    cfg = configs.config4(batch=4, M=8)
    n = net.ConvNet(cfg, max_norm=max_norm)
    n.set_inputs(cfg["inputs"](B=4), cfg["labels"](B=4))
    return n


@pytest.mark.parametrize("by_hand", [False, True])
def test_conv_network_steps_are_clipped(by_hand):
    """ConvNet(max_norm=...): step, and its parts called one by one."""
    c = 1e-3
    n = small_conv(c)
    if by_hand:
        n.forward()
        n.loss_grad()
        n.backward()
        n.optimizer()
    else:
        n.step()
    torch.cuda.synchronize()
    want, _ = norms(n.gW)
    assert want > c and n.grad_norm.item() == pytest.approx(want, rel=NORM)
    # the first step's m is (1 - beta1) of the clipped gradient: the factor, and a few roundings of each element
    m, _ = norms(n.m)
    assert m == pytest.approx(0.1 * c, rel=FACTOR + 8 * U)
    assert n.adam_state.tolist()[0] == 1


def test_dense_network_optimizer_by_hand_is_clipped():
    from paper_2607_14672_gb300 import configs, net
    cfg = configs.config2(batch=16, M=8)
    n = net.DenseNet(cfg, "x3", with_adamw=True, max_norm=1e-3)
    n.set_inputs(cfg["inputs"](B=16), cfg["labels"](B=16))
    n.forward_loss()
    n.backward()
    n.optimizer()
    torch.cuda.synchronize()
    m, _ = norms(n.m)
    assert m == pytest.approx(0.1 * 1e-3, rel=FACTOR + 8 * U)

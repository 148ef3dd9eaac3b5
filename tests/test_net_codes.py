"""The 8-bit weights of networks: handed from one to another, and needed before
anything is served (no GPU needed)."""

import pytest
import torch

from paper_2607_14672_gb300 import build, configs, net


@pytest.fixture(scope="module", autouse=True)
def lib():
    try:
        build.build()
    except RuntimeError:
        pytest.skip("the library does not build here")


def network(sizes, mode="q8", batch=2):
    cfg = configs.config2(batch=batch, M=8)
    layer = cfg["layers"][0]
    cfg["layers"] = [dict(layer, W=torch.zeros(b, a).numpy()) for a, b in zip(sizes, sizes[1:])]
    return net.DenseNet(cfg, mode, device="cpu")


def with_codes(n):
    for i, x in enumerate(n.Wq + n.w_scale):
        x.fill_(i + 1)
    n.has_codes = True
    return n


def test_codes_are_taken_over():
    a, b = with_codes(network((20, 30, 10))), network((20, 30, 10), batch=5)
    b.take_codes(a)
    assert b.has_codes
    assert all(torch.equal(x, y) for x, y in zip(a.Wq + a.w_scale, b.Wq + b.w_scale))


@pytest.mark.parametrize("sizes", [(20, 30), (20, 30, 10, 10), (20, 1, 10), (20, 30, 11), (1, 30, 10)])
def test_codes_of_other_layers_are_refused(sizes):
    """Fewer or more layers, or layers whose codes would be repeated to fit: nothing is taken."""
    a, b = with_codes(network(sizes)), network((20, 30, 10))
    for x in b.Wq + b.w_scale:
        x.fill_(-7)
    with pytest.raises(ValueError):
        b.take_codes(a)
    assert not b.has_codes and all((x == -7).all() for x in b.Wq + b.w_scale)


def test_nothing_is_served_or_taken_without_codes():
    a, b = network((20, 30, 10)), network((20, 30, 10))
    with pytest.raises(ValueError):
        b.take_codes(a)
    with pytest.raises(ValueError):
        b.take_codes(network((20, 30, 10), "x3"))
    with pytest.raises(RuntimeError):
        b.serve()
    with pytest.raises(RuntimeError):
        network((20, 30, 10), "x3").serve()

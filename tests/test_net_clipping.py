"""What a network's optimiser asks of the library, without a GPU."""

import pytest
import torch

from paper_2607_14672_gb300 import dstd, net


class Stub(net.Clipped):
    def __init__(self, max_norm):
        self.W = self.gW = self.m = self.v = [torch.zeros(3)]
        self.adam_state = torch.zeros(2, dtype=torch.int32)
        self.grad_norm, self.clip_workspace, self.max_norm = torch.zeros(1), None, max_norm


@pytest.fixture
def calls(monkeypatch):
    seen = []
    monkeypatch.setattr(dstd, "adamw_multi", lambda *a, **k: seen.append(None))
    monkeypatch.setattr(dstd, "adamw_clip", lambda *a, **k: seen.append(a[10]))
    return seen


def test_optimizer_clips_to_the_networks_norm(calls):
    Stub(0.5).optimizer()
    Stub(0.5).optimizer(lr=1e-2)
    Stub(0.5).optimizer(max_norm=2.0)
    Stub(0.5).optimizer(max_norm=None)          # without clipping, asked for
    Stub(None).optimizer()
    Stub(None).optimizer(max_norm=3.0)
    assert calls == [0.5, 0.5, 2.0, None, None, 3.0]


@pytest.mark.parametrize("kind", ["dense", "conv"])
def test_networks_with_an_optimiser_are_built_on_any_device(kind):
    """Their buffers need no GPU until a step runs."""
    from paper_2607_14672_gb300 import build, configs
    try:
        build.build()
    except RuntimeError:
        pytest.skip("the library does not build here")
    for max_norm in (None, 0.5):
        if kind == "dense":
            n = net.DenseNet(configs.config2(batch=4, M=8), "x3", device="cpu", with_adamw=True, max_norm=max_norm)
        else:
            n = net.ConvNet(configs.config4(batch=2, M=8), device="cpu", max_norm=max_norm)
        assert len(n.m) == len(n.W) and n.clip_workspace.numel() > 64 and not n.clip_workspace.any()


def test_launches_of_a_step_with_a_long_clipped_update():
    """A step of more than 2^24 weights forms its norm in a launch of its own."""
    from paper_2607_14672_gb300 import build, configs
    try:
        build.build()
    except RuntimeError:
        pytest.skip("the library does not build here")
    cfg = configs.config2(batch=4, M=8)
    cfg["layers"] = [dict(cfg["layers"][0], W=torch.zeros(4160, 4096).numpy())]
    plain, clipped = (net.DenseNet(cfg, "x3", device="cpu", with_adamw=True, max_norm=c).launches_per_step()
                      for c in (None, 0.5))
    assert clipped == plain + 1

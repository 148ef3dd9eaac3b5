"""Clipped steps of the networks, and gradients at the ends of the ranges, on the
GPU. Tolerances as derived in the tests of ordinary lists: NORM for the norm,
FACTOR for the clip factor."""

import math

import pytest
import torch

from test_gpu_clip import FACTOR, NORM, U, adamw_ref, host, lib, norms, workspace  # noqa: F401 (lib is a fixture)

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


def microseconds(f, n=10):
    for _ in range(3):
        f()
    times = []
    for _ in range(7):
        a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        a.record()
        for _ in range(n):
            f()
        b.record()
        torch.cuda.synchronize()
        times.append(a.elapsed_time(b) / n * 1e3)
    return sorted(times)[3]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_norm_of_zeros_takes_no_longer(dtype):
    """Gradients with rows of zeros, as silent neurons leave them, and of nothing
    else: the same bytes are read, so about the same time is taken (a factor of
    1.5 for the measurement), and the zeros count for nothing."""
    from paper_2607_14672_gb300 import dstd
    n = 1 << 26
    dense = torch.randn(n, device="cuda").to(dtype)
    rows = dense.clone()
    rows.view(-1, 4096)[::2] = 0
    rows.view(-1, 4096)[1::4] *= -0.0
    zeros = torch.zeros_like(dense)
    norm, ws = torch.empty(1, device="cuda"), workspace([dense])
    lists = [dstd.TensorList([x]) for x in (dense, rows, zeros)]
    took = [microseconds(lambda: dstd.grad_norm(l, norm, ws)) for l in lists]
    assert max(took[1:]) <= 1.5 * took[0], took
    assert norm.item() == 0.0
    dstd.grad_norm(lists[1], norm, ws)
    want = rows.double().square().sum().sqrt().item()
    assert norm.item() == pytest.approx(want, rel=NORM, abs=0)


@pytest.mark.parametrize("max_norm", [0.5, 1e-7, 1e-30])
@pytest.mark.parametrize("n", [1 << 18, (1 << 19) + 77])   # one launch, two launches
def test_clip_factors_below_fp32(n, max_norm):
    """max_norm / norm below fp32's normal numbers, or below its smallest one: the clipped gradients are as
    near as with any other factor."""
    from paper_2607_14672_gb300 import dstd
    g = torch.full((n,), 3e38, device="cuda")
    g[::2] = -1e38
    total, _ = norms([g])
    out, norm = torch.empty_like(g), torch.empty(1, device="cuda")
    dstd.clip_grads([g], max_norm, norm, workspace([g]), [out])
    want = host(g) * (max_norm / total)
    assert (abs(host(out) - want) <= (FACTOR + U) * abs(want)).all()


@pytest.mark.parametrize("n", [1 << 20, (1 << 24) + 5])   # one launch, two launches
def test_step_of_gradients_whose_norm_passes_fp32(n):
    """Finite gradients with a norm beyond fp32: norm[0] is inf, and the step is clipped, done and counted. One
    infinite gradient among them: norm[0] is inf as well, and nothing is done or counted."""
    from paper_2607_14672_gb300 import dstd
    lr, b1, b2, eps, wd, max_norm = 1e-3, 0.9, 0.999, 1e-8, 1e-2, 0.5
    g = torch.full((n,), 3e38, device="cuda")
    g[::2] = -1e38
    w, m, v = (torch.rand(n, device="cuda") * s for s in (0.1, 1e-2, 1e-6))
    before = [host(x) for x in (w, m, v)]
    step, norm, ws = torch.tensor([4], dtype=torch.int32, device="cuda"), torch.zeros(1, device="cuda"), workspace([g])
    dstd.adamw_clip([w], [g], [m], [v], lr, b1, b2, eps, wd, step, max_norm, norm, ws)
    total, _ = norms([g])
    assert total > 3.5e38 and norm.item() == math.inf and step.item() == 5
    w2, m2, v2, e_w, e_m, e_v = adamw_ref(before[0], host(g), before[1], before[2], 5, lr, b1, b2, eps, wd,
                                          max_norm / total)
    for got, want, off in ((w, w2, e_w), (m, m2, e_m), (v, v2, e_v)):
        assert (abs(host(got) - want) <= off).all()
    kept = [x.clone() for x in (w, m, v)]
    g[n // 3] = math.inf
    dstd.adamw_clip([w], [g], [m], [v], lr, b1, b2, eps, wd, step, max_norm, norm, ws)
    assert norm.item() == math.inf and step.item() == 5
    assert all(torch.equal(a, b) for a, b in zip((w, m, v), kept))

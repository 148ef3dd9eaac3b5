"""4-bit networks, and networks that learn from a teacher's record."""

import importlib.util
import math
import os

import numpy as np
import pytest
import torch

from oracle import distill as odistill
from oracle import dstd as odstd
from helpers import decode_saved, dense_layer, f32, grid_of, rel_l2

pytestmark = pytest.mark.gpu


def graph_of(n, state):
    """A captured step of n; the state is put back after the capture's first eager step."""
    keep = [x.clone() for x in state]
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        n.step(s)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        n.step(s)
    torch.cuda.synchronize()
    for x, b in zip(state, keep):
        x.copy_(b)
    torch.cuda.synchronize()
    return graph


def test_gradient_passes_straight_through():
    """dense_bwd at the 4-bit values and the 4-bit forward's spike state, against the oracle's backward there."""
    from paper_2607_14672_gb300 import dstd
    B, N_in, N_out, M = 6, 200, 300, 32
    t_in, layer = dense_layer(B, N_in, N_out, M, 0.5, 0.25, seed=4, t_offset=0.0)
    t_in, layer["W"] = f32(t_in), f32(layer["W"])
    p = dstd.params(layer, 1.0 / B)
    t, W = (torch.tensor(x, dtype=torch.float32, device="cuda") for x in (t_in, layer["W"]))
    q = torch.empty(N_out, dstd.mx4_row_bytes(N_in), dtype=torch.uint8, device="cuda")
    scale = torch.empty(dstd.mx4_scale_bytes(N_out, N_in), dtype=torch.uint8, device="cuda")
    Wv = torch.empty_like(W)
    dstd.quantize_mx4(W, q, scale, Wv)
    t_out, saved = torch.empty(B, N_out, device="cuda"), torch.empty(dstd.dense_saved_bytes(B, N_out), dtype=torch.uint8, device="cuda")
    ws = torch.empty(max(dstd.dense_mx4_workspace_bytes(B, N_in, N_out, p), dstd.dense_workspace_bytes(B, N_in, N_out, p, "x3")),
                     dtype=torch.uint8, device="cuda")
    dstd.dense_fwd_mx4(t, q, scale, p, t_out, saved, None, ws)
    g = torch.rand(B, N_out, device="cuda")
    g_t, g_W = torch.empty(B, N_in, device="cuda"), torch.empty(N_out, N_in, device="cuda")
    dstd.dense_bwd(t, Wv, t_out, saved, g, p, "x3", g_t, g_W, ws)
    torch.cuda.synchronize()
    bins, _, vdot = decode_saved(saved.cpu().numpy(), B, N_out)
    tg = t_out.cpu().numpy().astype(np.float64)
    assert 0.2 < np.isfinite(tg).mean()
    T, dt = grid_of(layer)
    ctx = dict(t=tg, q=bins.astype(int), vdot=vdot.astype(np.float64), fired=np.isfinite(tg),
               s=odstd.binning(t_in, T, dt, 0.5, 0.25))
    gW, gt, _ = odstd.backward_dense(ctx, t_in, Wv.cpu().numpy().astype(np.float64), g.cpu().numpy() * np.isfinite(tg),
                                     T, dt, 0.5, 0.25, 1.0)
    assert rel_l2(g_W.cpu().numpy(), gW) <= 1e-3 and rel_l2(g_t.cpu().numpy(), gt) <= 1e-3


def network(mode, B=32, **kw):
    from paper_2607_14672_gb300 import configs, net
    cfg = configs.config2(batch=B, M=16)
    n = net.DenseNet(cfg, mode, with_adamw=True, **kw)
    n.set_inputs(cfg["inputs"](B=B), cfg["labels"](B=B))
    return cfg, n


def record_of(n, K):
    top, index = torch.empty(n.B, K, device="cuda"), torch.empty(n.B, K, dtype=torch.int32, device="cuda")
    n.answers(top, index)
    return top, index


@pytest.mark.parametrize("mode", ["mx4", "x3", "bf16"])
@pytest.mark.parametrize("labels", [True, False])
def test_network_learns_from_a_record(mode, labels):
    """Loss and output gradient are those of the labels and of the record together; a captured step on records
    written in between gives what eager steps give."""
    from paper_2607_14672_gb300 import dstd
    cfg, n = network(mode, max_norm=0.5)
    _, teacher = network("x3")
    teacher.forward()
    top, index = record_of(teacher, 5)
    t = teacher.t[-1].cpu().numpy().astype(np.float64)
    factor, silent = -1.0 / cfg["tau_soft"], n.layers[-1]["t_end"]
    want = odistill.top_logits((np.float32(factor) * t.astype(np.float32)).astype(np.float64), 5, 1.0,
                               float(np.float32(factor) * np.float32(silent)))
    assert (index.cpu().numpy() == want[1]).all()
    index[3] = -1
    n.learn_from(5, weight=0.7, teacher_factor=0.5, labels=labels)
    n.set_teacher(top, index)

    def check(top, index):
        """Losses and the output gradient are those of the present output times."""
        torch.cuda.synchronize()
        value, rows, g = odistill.distill(n.t[-1].cpu().numpy(), top.cpu().numpy(), index.cpu().numpy(), factor, silent, 0.5, 0.7)
        assert abs(n.taught_loss[0].item() - value) <= 1e-5 * abs(value) and (rows == 0).sum() == 1
        ce, ce_g = torch.zeros(2, device="cuda"), torch.zeros_like(n.g[-1])
        dstd.ce_loss(n.t[-1], n.labels, cfg["tau_soft"], silent, ce, ce_g)
        torch.cuda.synchronize()
        if labels:
            g = g + ce_g.cpu().numpy()
            assert abs(n.loss[0].item() - ce[0].item()) <= 1e-5 * abs(ce[0].item())
        else:
            assert n.loss[0].item() == 0
        assert rel_l2(n.g[-1].cpu().numpy(), g) <= 1e-5
        return value

    n.forward_loss()
    check(top, index)
    assert abs(n.objective().item() - (n.loss[0] + n.taught_loss[0] + n.penalty[:, :2].sum()).item()) <= 1e-4
    # captured and eager steps on records written in between, from one state
    other = (top.flip(0).contiguous(), index.flip(0).contiguous())
    state = n.W + n.m + n.v + [n.adam_state]
    graph = graph_of(n, state)
    start = [x.clone() for x in state]
    values = []
    for step in (n.step, graph.replay):
        for r in (other, (top, index)):
            for x, b in zip(state, start):
                x.copy_(b)
            n.set_teacher(*r)
            torch.cuda.synchronize()
            step()
            values.append(check(*r))
            assert n.adam_state.tolist()[0] == 1 and not torch.equal(n.W[-1], start[len(n.W) - 1])
    assert abs(values[0] - values[1]) > 1e-3 and abs(values[2] - values[3]) > 1e-3


def test_network_serves_in_4_bits():
    """Serving on the kept codes gives the forward's times, and reads the codes alone."""
    _, n = network("mx4", max_norm=0.5)
    for _ in range(3):
        n.step()
    n.forward()
    times = [t.clone() for t in n.t]
    for w in n.W:
        w.fill_(math.nan)
    for t in n.t:
        t.zero_()
    n.serve()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(times, n.t))


def test_conv_network_learns_from_a_record():
    from paper_2607_14672_gb300 import configs, net
    cfg = configs.config4(batch=4)
    n = net.ConvNet(cfg, batch=4)
    n.set_inputs(cfg["inputs"](B=4), cfg["labels"](B=4))
    n.forward()
    top, index = record_of(n, 3)
    n.learn_from(3, labels=False)
    n.set_teacher(top * 0.25, index)
    n.step()
    torch.cuda.synchronize()
    factor, silent = -1.0 / cfg["tau_soft"], n.layers[-1]["t_end"]
    value, _, g = odistill.distill(n.t[-1].cpu().numpy(), (top * 0.25).cpu().numpy(), index.cpu().numpy(), factor, silent)
    assert abs(n.taught_loss[0].item() - value) <= 1e-5 * abs(value)
    assert rel_l2(n.g[-1].cpu().numpy(), g) <= 1e-5
    assert n.adam_state.tolist()[0] == 1


def test_example_distils_and_serves():
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "mx4_distill.py")
    spec = importlib.util.spec_from_file_location("mx4_distill", path)
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    losses, off = m.main(["--steps", "6", "--batch", "16"])
    assert all(math.isfinite(a) and math.isfinite(b) for a, b in losses)
    assert off <= 1e-4 * 1.2

"""The norm of many gradients, clipping and the clipped AdamW step on the GPU,
against the formulas in 64 bits.

How far the norm may be off: squares are added in fp32 in runs of at most 64
before they go into 64-bit sums, so the sum is within 65 * 2^-24 relative, the
norm within half of that plus its own fp32 rounding (NORM). The clip factor adds
one rounding, each product one more (FACTOR). AdamW's terms are bounded below
from those and a few roundings of 2^-24 each.
"""

import math

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
NORM = 65 * U / 2 + 2 * U
FACTOR = NORM + 2 * U
HALF = {torch.float32: U, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}   # one rounding to 24, 8, 11 bits


@pytest.fixture(scope="module", autouse=True)
def lib():
    from paper_2607_14672_gb300 import build, dstd
    build.build()
    dstd.load()
    assert dstd.device_status(clear=True) == 0
    yield
    assert dstd.device_status(clear=True) == 0


def tensors(sizes, types, seed, gap=0, size=1.0):
    """Tensors of one flat buffer per type, ``gap`` elements apart (odd gaps: not 16-byte aligned)."""
    g = np.random.default_rng(seed)
    out = []
    for i, n in enumerate(sizes):
        dt = types[i % len(types)]
        buf = torch.full((n + 2 * gap,), math.nan, dtype=dt, device="cuda")   # what must not count
        buf[gap:gap + n] = torch.tensor(g.normal(size=n) * size, dtype=torch.float64).to(dt)
        out.append(buf[gap:gap + n])
    return out


def host(x):
    return x.double().cpu().numpy()


def norms(gs):
    each = [float(np.sqrt((host(x) ** 2).sum())) for x in gs]
    return math.sqrt(sum(e * e for e in each)), each


def workspace(gs):
    from paper_2607_14672_gb300 import dstd
    return torch.zeros(dstd.grad_norm_workspace_bytes(gs), dtype=torch.uint8, device="cuda")


F, H, P = torch.float32, torch.bfloat16, torch.float16
LISTS = [((1,), (F,), 0), ((5,), (H,), 1), ((1000, 64, 4096), (F,), 0), ((1000, 63, 7), (F, H), 0),
         ((0, 17, 0, 1), (F, P), 0), ((0,), (F,), 0), ((1023, 1024, 1025, 2049), (F, H, P), 1),
         ((627200, 640000, 8000), (F,), 1), ((3000001, 5), (H,), 3), ((2500000, 1, 77), (F,), 0),
         (tuple(range(1, 41)), (H, F), 0), (tuple([3, 1500] * 300), (F, P), 1),
         ((17000001, 300), (H, F), 1), ((5,) * 200 + (900000,), (F,), 0)]


@pytest.mark.parametrize("sizes,types,gap", LISTS)
def test_grad_norm(sizes, types, gap):
    from paper_2607_14672_gb300 import dstd
    gs = tensors(sizes, types, len(sizes) + sizes[0], gap)
    norm, each = torch.full((1,), -1.0, device="cuda"), torch.full((len(gs),), -1.0, device="cuda")
    ws = workspace(gs)
    dstd.grad_norm(gs, norm, ws, each)
    alone = torch.empty(1, device="cuda")
    dstd.grad_norm(dstd.TensorList(gs), alone, ws)      # again on the same workspace, without the tensors' own
    torch.cuda.synchronize()
    want, want_each = norms(gs)
    assert norm.item() == pytest.approx(want, rel=NORM, abs=0)
    np.testing.assert_allclose(host(each), want_each, rtol=NORM, atol=0)
    assert alone.item() == norm.item()                  # the same bits every time
    assert not ws[:64].any()


@pytest.mark.parametrize("size", [1e-44, 1e-30, 1e-22, 1e-19, 1e15, 1e19, 1e25])
def test_grad_norm_beyond_fp32_squares(size):
    """Gradients whose squares leave fp32's range."""
    from paper_2607_14672_gb300 import dstd
    gs = tensors((5000, 33), (F,), 2, 0, size)
    norm = torch.empty(1, device="cuda")
    dstd.grad_norm(gs, norm, workspace(gs))
    torch.cuda.synchronize()
    want, _ = norms(gs)
    assert norm.item() == pytest.approx(want, rel=NORM, abs=2.0 ** -149)


@pytest.mark.parametrize("bad", [math.inf, -math.inf, math.nan])
@pytest.mark.parametrize("dtype", [F, H, P])
def test_not_finite(bad, dtype):
    """One infinite or NaN gradient: the norm shows it, gradients pass, a step changes nothing."""
    from paper_2607_14672_gb300 import dstd
    sizes = (700, 5001)
    gs = tensors(sizes, (dtype,), 9)
    gs[1][4000] = bad
    ws = workspace(gs)
    norm, each = torch.zeros(1, device="cuda"), torch.zeros(2, device="cuda")
    dstd.grad_norm(gs, norm, ws, each)
    assert not math.isfinite(norm.item()) and math.isfinite(each[0].item()) and not math.isfinite(each[1].item())
    outs = [torch.zeros_like(x) for x in gs]
    dstd.clip_grads(gs, 0.1, norm, ws, outs)
    assert not math.isfinite(norm.item())
    assert all(torch.equal(o.nan_to_num(5.0), x.nan_to_num(5.0)) for o, x in zip(outs, gs))
    w, m, v = ([torch.rand(n, device="cuda") for n in sizes] for _ in range(3))
    kept = [x.clone() for x in w + m + v]
    step = torch.tensor([3], dtype=torch.int32, device="cuda")
    dstd.adamw_clip(w, gs, m, v, 1e-3, 0.9, 0.999, 1e-8, 1e-2, step, 1.0, norm, ws)
    assert all(torch.equal(a, b) for a, b in zip(w + m + v, kept)) and step.item() == 3
    gs[1][4000] = 0.0                                   # and the next step works
    dstd.adamw_clip(w, gs, m, v, 1e-3, 0.9, 0.999, 1e-8, 1e-2, step, 1.0, norm, ws)
    assert step.item() == 4 and not torch.equal(w[0], kept[0])


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("max_norm", [0.25, 1e9, math.inf])
@pytest.mark.parametrize("sizes,types,gap", LISTS)
def test_clip_grads(sizes, types, gap, max_norm, in_place):
    from paper_2607_14672_gb300 import dstd
    gs = tensors(sizes, types, 3 + sizes[0], gap)
    g0 = [x.clone() for x in gs]
    outs = None if in_place else tensors(sizes, types, 1, gap)
    norm = torch.empty(1, device="cuda")
    dstd.clip_grads(gs, max_norm, norm, workspace(gs), outs)
    torch.cuda.synchronize()
    want, _ = norms(g0)
    assert norm.item() == pytest.approx(want, rel=NORM, abs=0)
    c = min(1.0, max_norm / want) if want > 0 else 1.0
    got = gs if in_place else outs
    for x, o in zip(g0, got):
        ref = host(x) * c
        if c == 1.0:
            assert torch.equal(o, x)
        else:  # fp16 results may be subnormal: half their step more
            np.testing.assert_allclose(host(o), ref, rtol=FACTOR + HALF[x.dtype] * (1 + 1e-3), atol=2.0 ** -25
                                       if x.dtype == P else 0)
    if not in_place:
        assert all(torch.equal(a, b) for a, b in zip(gs, g0))


def test_clip_grads_of_huge_gradients():
    """A norm past fp32 still clips: the factor is formed in 64 bits."""
    from paper_2607_14672_gb300 import dstd
    gs = [torch.full((1 << 20,), 3e38, device="cuda"), torch.full((3,), -1e38, device="cuda")]
    norm = torch.empty(1, device="cuda")
    dstd.clip_grads(gs, 1e36, norm, workspace(gs))
    assert norm.item() == math.inf
    total = math.sqrt((1 << 20) * float(np.float32(3e38)) ** 2 + 3 * float(np.float32(1e38)) ** 2)
    assert gs[0][77].item() == pytest.approx(float(np.float32(3e38)) * 1e36 / total, rel=FACTOR + U)


def adamw_ref(w, g, m, v, t, lr, b1, b2, eps, wd, c):
    """The step in 64 bits and how far fp32 may be off, element by element."""
    cg = c * g
    m2, v2 = b1 * m + (1 - b1) * cg, b2 * v + (1 - b2) * cg * cg
    e_g = (FACTOR + 2 * U) * np.abs((1 - b1) * cg)
    e_m = e_g + 4 * U * (np.abs(b1 * m) + np.abs((1 - b1) * cg))
    e_v = (2 * FACTOR + 4 * U) * (1 - b2) * cg * cg + 4 * U * v2 + 2.0 ** -140
    bc1, bc2 = 1 - b1 ** t, 1 - b2 ** t
    root = np.sqrt(v2 / bc2)
    den = root + eps
    e_root = np.minimum(0.5 * e_v / bc2 / np.maximum(root, 1e-300), np.sqrt(e_v / bc2)) + 6 * U * root
    u = lr * (m2 / bc1) / den
    # bias corrections: expm1 of a rounded t ln(beta), a few roundings
    e_u = lr * e_m / bc1 / den + np.abs(u) * ((e_root + U * den) / den + 12 * U)
    w2 = w * (1 - lr * wd) - u
    return w2, m2, v2, e_u + 4 * U * np.abs(w) + U * np.abs(w2), e_m, e_v


@pytest.mark.parametrize("sizes,types,gap", LISTS)
def test_adamw_clip(sizes, types, gap):
    from paper_2607_14672_gb300 import dstd
    lr, b1, b2, eps, wd, max_norm = 1e-3, 0.9, 0.999, 1e-8, 1e-2, 0.5
    ws_, ms = tensors(sizes, (F,), 5, gap, 0.1), tensors(sizes, (F,), 6, gap, 0.01)
    vs = [x.abs_() for x in tensors(sizes, (F,), 7, gap, 1e-4)]
    step = torch.tensor([0, 7], dtype=torch.int32, device="cuda")
    norm = torch.empty(1, device="cuda")
    for t in range(1, 4):
        gs = tensors(sizes, types, 100 + t, gap)
        g0 = [x.clone() for x in gs]
        before = [[host(x) for x in l] for l in (ws_, ms, vs)]
        dstd.adamw_clip(ws_, gs, ms, vs, lr, b1, b2, eps, wd, step, max_norm, norm, workspace(gs))
        torch.cuda.synchronize()
        want, _ = norms(gs)
        assert norm.item() == pytest.approx(want, rel=NORM, abs=0)
        assert step.tolist() == [t, 7]
        c = min(1.0, max_norm / want) if want > 0 else 1.0
        for i in range(len(sizes)):
            w2, m2, v2, e_w, e_m, e_v = adamw_ref(before[0][i], host(gs[i]), before[1][i], before[2][i], t, lr, b1, b2,
                                                  eps, wd, c)
            assert (np.abs(host(ms[i]) - m2) <= e_m).all()
            assert (np.abs(host(vs[i]) - v2) <= e_v).all()
            assert (np.abs(host(ws_[i]) - w2) <= e_w).all()
        assert all(torch.equal(a, b) for a, b in zip(gs, g0))


def test_adamw_clip_matches_adamw_multi_without_clipping():
    """max_norm = inf is the plain step; lr from device memory; under graph replay the count advances."""
    from paper_2607_14672_gb300 import dstd
    sizes = (4096, 63)
    a = [tensors(sizes, (F,), s, 0, 0.1) for s in (1, 2, 3)]
    a[2] = [x.abs_() for x in a[2]]
    b = [[x.clone() for x in l] for l in a]
    gs = tensors(sizes, (F,), 4)
    lr = torch.full((1,), 2e-3, device="cuda")
    step, step_b = torch.zeros(2, dtype=torch.int32, device="cuda"), torch.zeros(2, dtype=torch.int32, device="cuda")
    norm, ws = torch.empty(1, device="cuda"), workspace(gs)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        dstd.adamw_clip(a[0], gs, a[1], a[2], 1.0, 0.9, 0.999, 1e-8, 1e-2, step, math.inf, norm, ws, lr_dev=lr,
                        stream=s)
    for _ in range(3):
        graph.replay()
        dstd.adamw_multi(b[0], gs, b[1], b[2], 1.0, 0.9, 0.999, 1e-8, 1e-2, step_b, lr)
    torch.cuda.synchronize()
    assert step.tolist() == [3, 0]
    # adamw_multi forms 1 - beta2 and the bias corrections in fp32: 1e-5 relative
    for x, y in zip(a[0] + a[1] + a[2], b[0] + b[1] + b[2]):
        np.testing.assert_allclose(host(x), host(y), rtol=1e-4, atol=1e-6)


def test_workspace_serves_lists_of_any_size_in_turn():
    """One workspace, large enough for the longest list, used by lists that take
    different launches, in turn and twice over; its counters are left at zero."""
    from paper_2607_14672_gb300 import dstd
    lists = [tensors(s, (F,), 11 + i) for i, s in enumerate([(40,), (1000, 64), (20000000,), tuple([64] * 600)])]
    ws = torch.zeros(max(dstd.grad_norm_workspace_bytes(l) for l in lists), dtype=torch.uint8, device="cuda")
    norm = torch.empty(1, device="cuda")
    for _ in range(2):
        for l in lists:
            outs = [torch.empty_like(x) for x in l]
            dstd.clip_grads(l, 1.0, norm, ws, outs)
            want, _ = norms(l)
            assert norm.item() == pytest.approx(want, rel=NORM)
            got, _ = norms(outs)
            assert got == pytest.approx(1.0, rel=FACTOR + U)
            dstd.grad_norm(l, norm, ws)
            assert norm.item() == pytest.approx(want, rel=NORM)
            assert not ws[:64].any()


def test_lists_that_do_not_match_are_refused():
    from paper_2607_14672_gb300 import dstd
    g = tensors((10, 20), (F,), 1)
    ws, norm, step = workspace(g), torch.zeros(1, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    half = [x.bfloat16() for x in g]
    other = tensors((10, 21), (F,), 1)
    with pytest.raises(ValueError):
        dstd.clip_grads(g, 1.0, norm, ws, other)
    with pytest.raises(ValueError):
        dstd.clip_grads(g, 1.0, norm, ws, half)
    with pytest.raises(ValueError):
        dstd.adamw_clip(half, g, g, g, 1e-3, 0.9, 0.999, 1e-8, 0.0, step, 1.0, norm, ws)
    with pytest.raises(ValueError):
        dstd.adamw_clip(g, g, other, g, 1e-3, 0.9, 0.999, 1e-8, 0.0, step, 1.0, norm, ws)
    with pytest.raises(ValueError):
        dstd.grad_norm([g[0].view(2, 5).t()], norm, ws)
    with pytest.raises(dstd.DstdError):
        dstd.grad_norm(g, norm, ws[:64])


def test_network_steps_are_clipped():
    """DenseNet and the optimiser's max_norm: without it the step is the plain one."""
    from paper_2607_14672_gb300 import configs, net
    cfg = configs.config2(batch=16, M=8)
    nets = [net.DenseNet(cfg, "x3", with_adamw=True, max_norm=c) for c in (None, math.inf, 1e-3)]
    for n in nets:
        n.set_inputs(cfg["inputs"](B=16), cfg["labels"](B=16))
        n.step()
    torch.cuda.synchronize()
    want, _ = norms(nets[1].gW)
    assert nets[1].grad_norm.item() == pytest.approx(want, rel=NORM)
    # two backward passes differ in their atomics' order: where a gradient is nothing but that, the first step
    # may go the other way (2 lr), elsewhere hardly at all
    off = np.concatenate([np.abs(host(a) - host(b)).ravel() for a, b in zip(nets[0].W, nets[1].W)])
    assert off.max() <= 2.1e-3 and off.mean() <= 1e-5
    # the first step's m is (1 - beta1) of the clipped gradient
    m = math.sqrt(sum((host(x) ** 2).sum() for x in nets[2].m))
    assert m == pytest.approx(0.1 * 1e-3, rel=1e-4)

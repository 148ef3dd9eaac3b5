"""The largest logits of each row and the distillation loss, against the float64 oracle."""

import numpy as np
import pytest
import torch

from oracle import distill as oracle
from paper_2607_14672_gb300 import dstd

pytestmark = pytest.mark.gpu
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
HALF = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}
TINY = {"f32": 2.0 ** -126, "bf16": 2.0 ** -126, "f16": 2.0 ** -25}  # half the least step, where that counts
F32 = lambda v: float(np.float32(v))


def host(x):
    return x.detach().float().cpu().numpy().astype(np.float64)


def padded(rows, cols, pad, dtype, offset=0, fill=0):
    flat = torch.full((rows * (cols + pad) + offset + 1,), fill, dtype=dtype, device="cuda")
    return flat, flat[offset:offset + rows * (cols + pad)].view(rows, cols + pad)[:, :cols]


def top(y, K, **kw):
    R = y.shape[0]
    v, i = torch.empty(R, K, device="cuda"), torch.empty(R, K, dtype=torch.int32, device="cuda")
    dstd.top_logits(y, v, i, **kw)
    return v, i


def check_top(y, K, factor=1.0, silent=None):
    v, i = top(y, K, factor=factor, silent=silent)
    none = silent if silent is not None else (-np.inf if factor > 0 else np.inf)
    z = (np.float32(factor) * host(y).astype(np.float32)).astype(np.float64)   # logits are rounded to fp32 once
    want_v, want_i = oracle.top_logits(z, K, 1.0, float(np.float32(factor) * np.float32(none)))
    assert (i.cpu().numpy() == want_i).all()
    assert np.array_equal(host(v), want_v, equal_nan=True)


@pytest.mark.parametrize("type", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("R,C,pad,offset", [(1, 1, 0, 0), (3, 2, 0, 0), (9, 10, 0, 0), (5, 33, 1, 1), (4, 127, 0, 0),
                                            (3, 513, 3, 5), (2, 2048, 0, 0), (2, 2049, 5, 3), (3, 8192, 0, 0),
                                            (2, 8193, 1, 7), (2, 32768, 0, 0), (1, 131071, 0, 1)])
def test_top(type, R, C, pad, offset):
    gen = torch.Generator().manual_seed(C)
    _, y = padded(R, C, pad, TYPES[type], offset)
    y.copy_(torch.randn(R, C, generator=gen) * 2.5)
    for K in sorted({1, min(C, 2), min(C, 63), min(C, 256)}):
        check_top(y, K)
    check_top(y, min(C, 40), factor=-3.0)


def test_top_of_times():
    t = torch.rand(40, 10, generator=torch.Generator().manual_seed(1))
    t[torch.rand(40, 10, generator=torch.Generator().manual_seed(2)) < 0.3] = float("inf")
    t[3] = float("inf")
    check_top(t.cuda(), 4, -50.0, 1.2)
    check_top(t.cuda(), 10, -50.0)          # silent ones last, -inf, by class


@pytest.mark.parametrize("C", [5, 300, 2500, 9000, 40000])
def test_top_of_equal_rows(C):
    """All equal, nearly all equal, signed zeros, infinities and NaN: equal ones by ascending class."""
    y = torch.zeros(8, C)
    y[1, 1::2] = -0.0
    y[2] = -float("inf")
    y[3] = float("inf")
    y[4, C // 2] = float("nan")
    y[5] = 1.0
    y[5, C - 1], y[5, C // 3] = 2.0, 0.5
    y[6] = torch.arange(C) % 3
    y[7] = torch.arange(C, dtype=torch.float32)
    for K in sorted({1, 3, 5, min(C, 256)}):
        check_top(y.cuda(), K)
        check_top(y.bfloat16().cuda(), K)


@pytest.mark.parametrize("type", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("C", [32, 33, 64, 129, 255, 256, 257, 511, 1000, 1023, 1024, 1025])
def test_top_where_the_form_changes(type, C):
    """Random rows, rows of few different logits and rows with one that differs, at every alignment."""
    gen = torch.Generator().manual_seed(C)
    for offset in range(3):
        _, y = padded(10, C, 1 + offset, TYPES[type], offset)
        y.copy_(torch.randn(10, C, generator=gen) * 2.5)
        y[2] = y[2].sign()
        y[3] = (y[3] * 2).round()
        y[4], y[5], y[6] = 1.0, float("-inf"), -float("inf")
        y[4, C // 2], y[5, C - 1], y[5, 0] = 2.0, 0.5, float("nan")
        y[7, :: 2] = -0.0
        y[7, 1:: 2] = 0.0
        y[8].copy_(torch.arange(C) * -1e-3)
        y[9].copy_(torch.randn(C, generator=gen).clamp(max=0.0))
        for K in sorted({1, min(C, 24), min(C, 25), 32, min(C, 33), min(C, 57), min(C, 64), min(C, 65)}):
            check_top(y, K)
        check_top(y, 20, factor=-3.0)
        check_top(y, min(C, 50), -50.0, 1.2)
        _, many = padded(800, C, 1 + offset, TYPES[type], offset)
        many.copy_(y.repeat(80, 1))
        for K, kw in [(1, {}), (24, {}), (min(C, 33), {}), (min(C, 64), {}), (min(C, 65), {}), (min(C, 100), {}), (min(C, 128), {}), (20, dict(factor=-3.0)), (min(C, 50), dict(factor=-50.0, silent=1.2))]:
            for few, all in zip(top(y, K, **kw), top(many, K, **kw)):
                assert torch.equal(few.repeat(80, 1).view(torch.int32), all.view(torch.int32))


def make(R, C, K, type, seed=0, pad=0, offset=0, times=False, gpad=0, goffset=0):
    gen = torch.Generator().manual_seed(seed)
    _, y = padded(R, C, pad, TYPES[type], offset)
    if times:
        t = torch.rand(R, C, generator=gen) * 0.2 + 0.8
        t[torch.rand(R, C, generator=gen) < 0.1] = float("inf")
        y.copy_(t)
    else:
        y.copy_(torch.randn(R, C, generator=gen) * 2.5)
    v = torch.randn(R, K, generator=gen) * 2
    i = torch.randint(0, C, (R, K), generator=gen, dtype=torch.int32)
    i[torch.rand(R, K, generator=gen) < 0.1] = -1
    return y, v.cuda(), i.cuda(), padded(R, C, gpad, TYPES[type], goffset, fill=3)


def close(got, want, size, type, steps):
    """One rounding of the type, and `steps` roundings of fp32 of `size`."""
    off = np.abs(got - want)
    allow = HALF[type] * np.abs(want) + steps * 2.0 ** -24 * size + TINY[type]
    assert (off <= allow).all(), (off / allow).max()


def check(y, v, i, g, type, factor=1.0, silent=None, teacher_factor=1.0, weight=1.0, row_weight=None, accumulate=False):
    R, C = y.shape
    flat, grad = g
    loss, rows = torch.zeros(2, device="cuda"), torch.full((R,), 9.0, device="cuda")
    before = host(grad)
    dstd.distill_loss(y, v, i, loss, rows, grad, factor, silent, teacher_factor, weight, row_weight, accumulate)
    none = silent if silent is not None else (-np.inf if factor > 0 else np.inf)
    f = F32(factor)
    want, want_rows, want_g = oracle.distill(host(y), host(v), i.cpu().numpy(), f, F32(none), F32(teacher_factor),
                                             F32(weight), None if row_weight is None else host(row_weight))
    z, silent_at = oracle.logits(host(y), f, F32(none))
    zt = F32(teacher_factor) * host(v)
    # exponents carry the roundings of logits of this size (each logit and each difference of two rounded to
    # fp32, exp and log to a few units), the sum one addition in its tree or chain for each of a thread's columns
    reach = 8 + 4 * (np.abs(z[np.isfinite(z)]).max(initial=0) + np.abs(zt[np.isfinite(zt)]).max(initial=0)) + C / 256 + i.shape[1] / 32
    if type != "f32":
        reach += 64                                     # the fast exp: 2^-21 and 2^-24 of its argument
    w = np.full(R, 1.0 / R) if row_weight is None else host(row_weight)
    q = np.exp(z - np.maximum(z.max(1, keepdims=True), -1e300))
    q /= np.maximum(q.sum(1, keepdims=True), 1e-300)
    mass = np.zeros_like(q)
    for r in range(R):
        used = [k for k in range(v.shape[1]) if 0 <= i[r, k] < C and zt[r, k] != -np.inf]
        if used:
            p = np.exp(zt[r, used] - zt[r, used].max())
            np.add.at(mass[r], i[r].cpu().numpy()[used], p / p.sum())
    size = np.abs(weight * w * f)[:, None] * (q + mass) * reach
    if accumulate:
        close(host(grad), before + want_g, size + np.abs(before), type, 1)
    else:
        close(host(grad), want_g, size, type, 1)
    assert (host(grad)[silent_at] == (before[silent_at] if accumulate else 0)).all()
    close(host(rows), want_rows, reach * (1 + np.abs(want_rows)), "f32", 4)
    close(host(loss)[:1], np.array([want]), abs(weight) * np.sum(np.abs(w) * reach * (1 + np.abs(want_rows))), "f32", 4)
    assert loss[1].item() == 0
    alone = torch.zeros(2, device="cuda")
    dstd.distill_loss(y, v, i, alone, torch.empty(R, device="cuda"), None, factor, silent, teacher_factor, weight, row_weight)
    assert torch.equal(alone, loss)
    pad = torch.ones_like(flat, dtype=torch.bool)
    torch.as_strided(pad, grad.shape, grad.stride(), grad.storage_offset()).fill_(False)
    assert (flat[pad] == 3).all()


@pytest.mark.parametrize("type", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("R,C,K", [(1, 1, 1), (3, 2, 2), (256, 10, 4), (17, 33, 20), (9, 129, 64), (5, 1000, 64), (5, 1000, 65),
                                   (3, 1025, 7), (4, 5000, 128), (3, 8193, 256), (2, 32768, 64), (1, 131071, 100)])
def test_distill(type, R, C, K):
    y, v, i, g = make(R, C, K, type, seed=C)
    check(y, v, i, g, type)


@pytest.mark.parametrize("type", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("C", [64, 65, 256, 257, 511, 512, 513, 1024, 2047, 2048, 2049, 9000])
def test_sizes_where_the_form_changes(type, C):
    y, v, i, g = make(11, C, 33, type, C, pad=1, gpad=1)
    check(y, v, i, g, type)
    check(y, v, i, g, type, factor=-0.5)
    y, v, i, g = make(4, C, 64, type, C, times=True)
    check(y, v, i, g, type, factor=-50.0, silent=1.2, weight=2.0)


@pytest.mark.parametrize("type,C,K", [("f32", 65, 65), ("bf16", 300, 128), ("f16", 1000, 97), ("f32", 1024, 128)])
def test_many_rows_of_long_records(type, C, K):
    y, v, i, g = make(700, C, K, type, seed=C, pad=1, offset=1)
    check(y, v, i, g, type)
    i[:, K // 2:] = i[:, :K - K // 2].clone()          # and classes named twice
    check(y, v, i, g, type)


def test_many_rows():
    """More rows than blocks at a time, each form; the sum over them."""
    for C, K in ((12, 4), (200, 6), (900, 20), (3000, 70)):
        y, v, i, g = make(5000, C, K, "bf16", C)
        loss, rows = torch.zeros(2, device="cuda"), torch.empty(5000, device="cuda")
        w = torch.rand(5000, device="cuda")
        dstd.distill_loss(y, v, i, loss, rows, g[1], row_weight=w, weight=0.5)
        want = 0.5 * (w.double() * rows.double()).sum().item()
        # a rounding of each product and of the compensated sums, and a tree of 8 or 9 levels
        assert abs(loss[0].item() - want) <= 12 * 2.0 ** -24 * 0.5 * (w.double() * rows.double().abs()).sum().item()
        few = slice(4990, 5000)
        loss2, rows2 = torch.zeros(2, device="cuda"), torch.empty(10, device="cuda")
        g2 = torch.empty_like(g[1][few])
        dstd.distill_loss(y[few], v[few], i[few], loss2, rows2, g2, row_weight=w[few], weight=0.5)
        assert torch.equal(rows[few], rows2) and torch.equal(g[1][few], g2)


@pytest.mark.parametrize("type", ["f32", "bf16"])
@pytest.mark.parametrize("pad,offset,gpad,goffset", [(1, 0, 0, 0), (0, 1, 0, 1), (3, 5, 8, 2), (4, 4, 4, 4), (8, 3, 8, 3)])
@pytest.mark.parametrize("C", [10, 77, 1500, 9001])
def test_strides_and_alignment(type, C, pad, offset, gpad, goffset):
    y, v, i, g = make(6, C, 9, type, C, pad, offset, False, gpad, goffset)
    check(y, v, i, g, type)
    check(y, v, i, g, type, accumulate=True)


@pytest.mark.parametrize("C", [3, 10, 700, 3000])
def test_times(C):
    y, v, i, g = make(19, C, 6, "f32", 5, times=True)
    check(y, v, i, g, "f32", factor=-50.0, silent=1.2, teacher_factor=0.5, weight=4.0)


@pytest.mark.parametrize("C,K", [(10, 40), (600, 64), (600, 200), (9000, 256)])
def test_the_same_class_several_times(C, K):
    y, v, i, g = make(5, C, K, "f32", 7)
    i[:, :] = i % 7
    i[2] = 4
    check(y, v, i, g, "f32")
    check(y, v, i, g, "f32", accumulate=True)


@pytest.mark.parametrize("C", [10, 1200, 9000])
def test_rows_left_out(C):
    """No teacher, classes out of range, no logits, no weight: loss and gradient are 0."""
    y, v, i, (flat, g) = make(8, C, 4, "f32", 3)
    i[0] = -1
    i[1] = torch.tensor([C, C + 5, -7, 2 ** 31 - 1])
    v[2] = -float("inf")
    y[3] = -float("inf")
    w = torch.rand(8, device="cuda")
    w[4] = 0
    y[5, 1] = -float("inf")
    i[5] = torch.tensor([0, 2, 2, -1])
    check(y, v, i, (flat, g), "f32", row_weight=w)
    assert (g[:5] == 0).all()
    g.fill_(2.0)
    dstd.distill_loss(y, v, i, torch.zeros(2, device="cuda"), torch.empty(8, device="cuda"), g, row_weight=w, accumulate=True)
    assert (g[:5] == 2).all() and (g[5:] != 2).any(1).all()


@pytest.mark.parametrize("C", [10, 1200, 9000, 40000])
def test_values_that_are_not_finite(C):
    y, v, i, (flat, g) = make(5, C, 3, "f32", 3)
    i[:] = torch.tensor([0, 1, 2])
    y[0, 2], y[1, 3], v[2, 1] = float("nan"), float("inf"), float("nan")
    y[3, 1] = -float("inf")                  # the teacher's class is masked: an infinite loss, and no gradient there
    loss, rows = torch.zeros(2, device="cuda"), torch.zeros(5, device="cuda")
    dstd.distill_loss(y, v, i, loss, rows, g)
    r = host(rows)
    assert np.isnan(r[:3]).all() and r[3] == np.inf and np.isfinite(r[4])
    gh = host(g)
    assert np.isnan(gh[0]).any() and np.isnan(gh[1]).any() and np.isnan(gh[2, :3]).all() and np.isfinite(gh[2, 3:]).all()
    assert np.isfinite(gh[3:]).all() and gh[3, 1] == 0
    assert loss[1].item() == 0


def test_long_rows_of_far_logits():
    """Logits that spread over hundreds, ascending and descending: the running maximum is rescaled throughout."""
    C = 20000
    y = torch.stack([torch.linspace(-300, 300, C), torch.linspace(300, -300, C), torch.full((C,), -80.0)]).cuda()
    v, i = top(y, 8)
    g = padded(3, C, 0, torch.float32, fill=3)
    check(y, v * 0.5, i, g, "f32")


def test_distill_gradient_against_differences():
    y, v, i, (_, g) = make(3, 7, 4, "f32", 11)
    loss, rows = torch.zeros(2, device="cuda"), torch.zeros(3, device="cuda")
    dstd.distill_loss(y, v, i, loss, rows, g, factor=0.7, weight=2.0)
    for r in range(3):
        for c in range(7):
            d = []
            for h in (2.0 ** -6, -2.0 ** -6):
                z = y.clone()
                z[r, c] += h
                dstd.distill_loss(z, v, i, loss, rows, None, factor=0.7, weight=2.0)
                d.append(rows.double().sum().item() * 2.0 / 3.0)
            # third derivative of the loss below 2 (weight factor^3 / 3), and fp32 losses of size 10
            assert abs((d[0] - d[1]) / 2.0 ** -5 - g[r, c].item()) < 2.0 ** -12 + 20 * 2.0 ** -24 * 2 ** 5


def test_same_bits_and_a_graph():
    y, v, i, (_, g) = make(300, 500, 16, "bf16", 4)
    loss, rows = torch.zeros(2, device="cuda"), torch.empty(300, device="cuda")
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    tv, ti = torch.empty(300, 16, device="cuda"), torch.empty(300, 16, dtype=torch.int32, device="cuda")
    with torch.cuda.stream(stream):
        dstd.top_logits(y, tv, ti)
        dstd.distill_loss(y, tv, ti, loss, rows, g)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        dstd.top_logits(y, tv, ti, stream=stream)
        dstd.distill_loss(y, v, i, loss, rows, g, stream=stream)
    seen = []
    for _ in range(3):
        g.fill_(0)
        graph.replay()
        torch.cuda.synchronize()
        seen.append((loss.clone(), rows.clone(), g.clone()))
    for a in seen[1:]:
        assert all(torch.equal(p, q) for p, q in zip(a, seen[0]))
    eager = torch.zeros(2, device="cuda")
    dstd.distill_loss(y, v, i, eager, rows, g)
    assert torch.equal(eager, seen[0][0])


# -- logits far from 0 ---------------------------------------------------------
def check_near(y, v, i, g, type, factor, w):
    """Factors of a power of two, so that logits and near differences are exact in fp32: nothing may grow with |z|, only
    with the distance from the row's largest. In units of 2^-24: an exponential's argument has up to four roundings of its
    size (the difference, log2(e), two products), the exponential itself 4 (2^-22); a sum adds its terms' own, a rescaling
    (one exponential and a product) and an addition for each batch of a thread's columns, and 16 for the trees and
    the division; a log and the sums of the loss 8. exp below 2^-126 may count as 0."""
    R, C = y.shape
    K = v.shape[1]
    loss, rows = torch.zeros(2, device="cuda"), torch.full((R,), 9.0, device="cuda")
    dstd.distill_loss(y, v, i, loss, rows, g, factor, row_weight=w)
    index, zt, wh = i.cpu().numpy(), host(v), host(w)
    want, want_rows, want_g = oracle.distill(host(y), zt, index, factor, row_weight=wh)
    z = factor * host(y)
    gap = z.max(1, keepdims=True) - z
    e = np.exp(-gap)
    q = e / e.sum(1, keepdims=True)
    far = np.where(q > 0, gap, 0.0)
    sums = (q * 4 * far).sum(1) + 24 + 3 * C / 256
    gt = zt.max(1, keepdims=True) - zt
    p = np.exp(-gt) / np.exp(-gt).sum(1, keepdims=True)
    of_p = 4 * gt + (p * 4 * gt).sum(1, keepdims=True) + 24 + K / 16
    mass, of_mass = np.zeros((R, C)), np.zeros((R, C))
    at = np.arange(R)[:, None].repeat(K, 1)
    np.add.at(mass, (at, index), p)
    np.add.at(of_mass, (at, index), p * (of_p + K / 16))
    u = 2.0 ** -24
    allow = HALF[type] * np.abs(want_g) + u * np.abs(wh * factor)[:, None] * (q * (4 * far + sums[:, None] + 8) + of_mass + 4 * mass)
    off = np.abs(host(g) - want_g)
    assert (off <= allow + TINY[type]).all(), (off / (allow + TINY[type])).max()
    gap_k = np.take_along_axis(gap, index, 1)
    log_s = np.log(e.sum(1))
    apart = np.abs(np.log(p) + gap_k + log_s[:, None])
    allow = u * ((p * ((of_p + 8) * (apart + 1) + 4 * (gt + gap_k))).sum(1) + sums + 8 * (log_s + 1) + 8 * np.abs(want_rows))
    off = np.abs(host(rows) - want_rows)
    assert (off <= allow).all(), (off / allow).max()
    whole = (wh * (allow + 4 * u * np.abs(want_rows))).sum()
    assert abs(loss[0].item() - want) <= whole and loss[1].item() == 0


# sizes of every form: a warp to a row (single columns, packs), a block, blocks of a cluster, many rows of a block each
FORMS = [(6, 10, 4), (6, 300, 9), (6, 1000, 64), (6, 3000, 7), (6, 9000, 100), (6, 40000, 30), (650, 1000, 100), (800, 3000, 5)]


@pytest.mark.parametrize("type", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("R,C,K", FORMS)
@pytest.mark.parametrize("factor", [1.0, -0.5])
def test_logits_far_from_zero(type, R, C, K, factor):
    """A common offset changes nothing but the inputs' own rounding."""
    for offset in (50.0, -1000.0, 30000.0):
        y, v, i, (_, g) = make(R, C, K, type, seed=C, pad=1)
        y.copy_(y.float() + offset)
        check_near(y, v, i.clamp_(min=0), g, type, factor, torch.full((R,), 1.0 / R, device="cuda"))


@pytest.mark.parametrize("type", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("R,C,K", FORMS)
@pytest.mark.parametrize("factor", [1.0, -1.0])
def test_logits_at_the_types_ends(type, R, C, K, factor):
    """Classes masked with the type's lowest value: all of a row's, all but one; rows at the largest value and near it."""
    y, v, i, (_, g) = make(R, C, K, type, seed=C + 1, pad=1)
    i.clamp_(min=0)
    end = torch.finfo(TYPES[type]).max
    z = y.float() * factor
    z[0] = -end
    z[1] = -end
    z[1, C // 2] = 1.0
    i[1] = C // 2
    z[2] = end
    z[3] = end * 0.75
    z[3, C - 1] = end * 0.5
    i[3] = 0
    z[4, 1::2] = -end
    i[4] = torch.arange(K) % ((C + 1) // 2) * 2
    z[5, :] = end
    z[5, ::3] = end * (1 - 2.0 ** -6)
    i[5] = torch.arange(K) % (C // 3) * 3 + 1
    y.copy_(z * factor)
    check_near(y, v, i, g, type, factor, torch.full((R,), 1.0 / R, device="cuda"))


@pytest.mark.parametrize("type,factor", [("bf16", 2.0 ** -126), ("bf16", 2.0 ** -119), ("f16", 2.0 ** -15)])
@pytest.mark.parametrize("C", [300, 9000])
def test_smallest_factors(type, factor, C):
    """Outputs at both ends of the type whose logits lie near each other, for their factor is small."""
    y, v, i, (_, g) = make(5, C, 6, type, seed=C)
    i.clamp_(min=0)
    end = torch.finfo(TYPES[type]).max
    y.copy_((y.float() * 0.2).clamp(-1, 1) * end)
    y[0, 0], y[0, 1] = end, -end
    check_near(y, v, i, g, type, factor, torch.ones(5, device="cuda"))


@pytest.mark.parametrize("type", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("C", [10, 300, 1200, 9000, 40000])
@pytest.mark.parametrize("factor", [1.0, -1.0])
def test_masked_classes_of_rows_that_are_not_finite(type, C, factor):
    """A masked class passes no gradient, whatever else its row holds: 0 written, nothing added."""
    y, v, i, (_, g) = make(6, C, 3, type, 3, pad=1)
    i[:] = torch.tensor([0, 1, 2])
    masked = torch.zeros(6, C, dtype=torch.bool, device="cuda")
    masked[:, 5::3] = True
    masked[5] = True
    y[masked] = -float("inf") * factor
    y[0, 3], y[1, 3], v[2, 1] = float("nan"), float("inf") * factor, float("nan")
    y[5, 4] = float("nan")                   # nothing but masked classes and a NaN
    w = torch.full((6,), 0.25, device="cuda")
    w[3] = float("nan")
    loss, rows = torch.zeros(2, device="cuda"), torch.zeros(6, device="cuda")
    for accumulate in (False, True):
        g.fill_(3.0)
        dstd.distill_loss(y, v, i, loss, rows, g, factor, row_weight=w, accumulate=accumulate)
        assert (g[masked] == (3.0 if accumulate else 0.0))[~torch.isnan(y[masked])].all()
        for r in (0, 1, 3):
            assert torch.isnan(g[r][~masked[r]]).all()
        assert torch.isnan(g[5, 4]) and torch.isnan(g[2, :3]).all() and torch.isfinite(g[2, 3:]).all()
        assert torch.isfinite(g[4]).all()
        assert torch.isnan(rows[[0, 1, 2, 5]]).all() and torch.isfinite(rows[[3, 4]]).all() and torch.isnan(loss[0])


@pytest.mark.parametrize("type", ["bf16", "f16"])
@pytest.mark.parametrize("C", [10, 300, 1200, 9000, 40000])
def test_rows_left_out_in_16_bits(type, C):
    """As in fp32: no teacher, classes out of range, no logits, no weight, masked classes named."""
    y, v, i, (flat, g) = make(8, C, 4, type, 3)
    i[0] = -1
    i[1] = torch.tensor([C, C + 5, -7, 2 ** 31 - 1])
    v[2] = -float("inf")
    y[3] = -float("inf")
    w = torch.linspace(0.5, 1, 8, device="cuda")
    w[4] = 0
    y[5, 1::2] = -float("inf")
    i[5] = torch.tensor([0, 2, 2, -1])
    check(y, v, i, (flat, g), type, row_weight=w)
    assert (g[:5] == 0).all()
    g.fill_(2.0)
    dstd.distill_loss(y, v, i, torch.zeros(2, device="cuda"), torch.empty(8, device="cuda"), g, row_weight=w, accumulate=True)
    assert (g[:5] == 2).all() and (g[5:] != 2).any(1).all()


@pytest.mark.parametrize("type", ["bf16", "f16"])
@pytest.mark.parametrize("C,K", [(10, 40), (300, 64), (600, 200), (9000, 256), (40000, 100)])
def test_the_same_class_several_times_in_16_bits(type, C, K):
    y, v, i, g = make(5, C, K, type, 7)
    i[:, :] = i % 7
    i[2] = 4
    y[3, 1::3] = -float("inf")
    i[3] = i[3] // 3 * 3
    check(y, v, i, g, type)
    check(y, v, i, g, type, accumulate=True)

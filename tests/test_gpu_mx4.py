"""4-bit rows, their products and the layer forward on them, against the float64 oracle."""

import numpy as np
import pytest
import torch

from mx4_plans import PLANS
from oracle import mx4
from paper_2607_14672_gb300 import dstd

pytestmark = pytest.mark.gpu
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


def host(x):
    return x.detach().float().cpu().numpy().astype(np.float64)


def padded(rows, cols, pad, dtype, offset=0, fill=0):
    """A matrix with `pad` more elements to a row, `offset` elements into its storage; the padding holds `fill`."""
    flat = torch.full((rows * (cols + pad) + offset + 1,), fill, dtype=dtype, device="cuda")
    return flat, flat[offset:offset + rows * (cols + pad)].view(rows, cols + pad)[:, :cols]


def quantized(x, values=False, pad=0):
    R, K = x.shape
    row = dstd.mx4_row_bytes(K)
    _, q = padded(R, row, 16 * pad, torch.uint8, fill=0xEE)
    scale = torch.full((dstd.mx4_scale_bytes(R, K),), 0xEE, dtype=torch.uint8, device="cuda")
    v = torch.empty(R, K, device="cuda") if values else None
    dstd.quantize_mx4(x, q, scale, v)
    return q, scale, v


def decoded(q, scale, K):
    return mx4.value_of(*mx4.unpack(q.cpu().numpy(), scale.cpu().numpy(), K))


@pytest.mark.parametrize("type", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("R,K,pad,offset", [(1, 1, 0, 0), (3, 31, 0, 0), (2, 32, 0, 0), (5, 33, 3, 1), (130, 128, 0, 0),
                                            (129, 129, 7, 5), (4, 1000, 8, 0), (2, 4097, 1, 3), (261, 300, 4, 4)])
def test_quantize(type, R, K, pad, offset):
    gen = torch.Generator().manual_seed(R * 1000 + K)
    x = torch.randn(R, K, generator=gen) * 10.0 ** (torch.rand(R, K, generator=gen) * 3 - 2)
    x[torch.rand(R, K, generator=gen) < 0.2] = 0
    _, xd = padded(R, K, pad, TYPES[type], offset)
    xd.copy_(x)
    row = dstd.mx4_row_bytes(K)
    flat, q = padded(R, row, 16, torch.uint8, fill=0xEE)
    scale = torch.full((dstd.mx4_scale_bytes(R, K) + 16,), 0xEE, dtype=torch.uint8, device="cuda")
    vflat, v = padded(R, K, pad, torch.float32, offset, fill=7)
    dstd.quantize_mx4(xd, q, scale, v)
    codes, e, values = mx4.quantize(host(xd))
    want_q, want_s = mx4.pack(codes, e)
    assert (q.cpu().numpy() == want_q).all()
    got_s = scale.cpu().numpy()
    n = mx4.blocks_of(K)
    r, b = np.arange(R)[:, None], np.arange(-(-n // 4) * 4)[None, :]
    at = mx4.scale_place(r, b, K)
    assert (got_s[at] == want_s[at]).all()      # those of blocks past the last are 0
    assert (host(v) == values).all()
    # nothing else is written
    if K:
        assert (got_s[-16:] == 0xEE).all()
    mine = torch.zeros_like(flat, dtype=torch.bool)
    mine[:R * (row + 16)].view(R, row + 16)[:, :row] = True
    assert (flat[~mine] == 0xEE).all()
    mine = torch.zeros_like(vflat, dtype=torch.bool)
    mine[offset:offset + R * (K + pad)].view(R, K + pad)[:, :K] = True
    assert (vflat[~mine] == 7).all()


@pytest.mark.parametrize("type", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("R,K,pad,offset", [(20000, 130, 0, 0), (20000, 260, 4, 4), (40000, 500, 12, 0), (40000, 1000, 1, 3),
                                            (12000, 1024, 0, 0), (9000, 5000, 0, 1), (80000, 250, 6, 2)])
def test_many_rows(type, R, K, pad, offset):
    """Many rows take several runs of a row to a warp: the same bytes as in slices of few, which take one."""
    gen = torch.Generator(device="cuda").manual_seed(K)
    _, x = padded(R, K, pad, TYPES[type], offset)
    x.copy_(torch.randn(R, K, generator=gen, device="cuda") * torch.exp2(torch.randn(R, K, generator=gen, device="cuda") * 4))
    x[5, K // 2], x[R - 1, K - 1] = float("inf"), float("nan")
    q, scale, v = quantized(x, True)
    plain, scale2, _ = quantized(x)
    assert torch.equal(q, plain)
    n = mx4.blocks_of(K)
    for i in [0, 128 * 7, (R - 1) // 128 * 128]:
        few = x[i:i + 128]
        q1, s1, v1 = quantized(few, True)
        assert torch.equal(q[i:i + 128], q1) and torch.equal(v[i:i + 128].nan_to_num(7.0), v1.nan_to_num(7.0))
        r, b = np.arange(few.shape[0])[:, None], np.arange(-(-n // 4) * 4)[None, :]
        mine, all = mx4.scale_place(r, b, K), mx4.scale_place(r + i, b, K)
        for s in (scale, scale2):
            assert (s.cpu().numpy()[all] == s1.cpu().numpy()[mine]).all()
    # every row: the widest step, from 4 to 6, is off by at most 1, and 2^e is at most a third of the largest
    fine = torch.isfinite(v)
    wide = torch.nn.functional.pad(torch.isfinite(x), (0, -K % 32), value=True).view(R, n, 32)
    assert torch.equal(fine, wide.all(2).repeat_interleave(32, 1)[:, :K]) and not fine.all()
    d = (v.double() - x.double()).abs()[fine]
    top = torch.nn.functional.pad(x.double(), (0, -K % 32)).view(R, n, 32).abs().amax(2).repeat_interleave(32, 1)[:, :K]
    assert (d <= (top / 3)[fine]).all()


def test_quantize_edges():
    """Ties, the ends of fp32, signed zeros, and blocks that are not finite."""
    x = torch.zeros(6, 96)
    x[0, :11] = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0, -0.25, -5.0, -0.75])
    x[1, :4] = torch.tensor([3.4e38, -3.4e38, 1e38, 1e-45])
    x[2, :4] = torch.tensor([1e-45, -1e-44, 3e-39, -0.0])
    x[3, 5], x[3, 40] = float("inf"), 1.0
    x[4, 37], x[4, 3] = float("nan"), 2.0
    x[5, 70] = -float("inf")
    q, scale, v = quantized(x.cuda(), True)
    codes, e, values = mx4.quantize(x.numpy())
    assert (q.cpu().numpy() == mx4.pack(codes, e)[0]).all()
    with np.errstate(over="ignore"):
        values = values.astype(np.float32).astype(np.float64)     # 3.4e38 is nearest to 2^128, past fp32
    assert np.isinf(values).sum() == 2
    got = host(v)
    assert np.array_equal(np.isnan(got), np.isnan(values)) and np.isnan(values).sum() == 96
    assert (got[~np.isnan(values)] == values[~np.isnan(values)]).all()
    assert np.isnan(decoded(q, scale, 96)).sum() == 96


def test_quantize_nothing():
    q = torch.empty(0, 16, dtype=torch.uint8, device="cuda")
    s = torch.empty(0, dtype=torch.uint8, device="cuda")
    dstd.quantize_mx4(torch.empty(0, 20, device="cuda"), q, s)
    dstd.quantize_mx4(torch.empty(3, 0, device="cuda"), torch.empty(3, 0, dtype=torch.uint8, device="cuda"), s)
    torch.cuda.synchronize()


def bound(x, w, out):
    """A sum of blocks is formed in fp32, each block of 32 products and each addition off by at most
    2^-23 of the magnitudes summed so far; one more rounding to 16 bits."""
    n = mx4.blocks_of(x.shape[1])
    size = np.abs(x) @ np.abs(w).T
    eps = {"f32": 0.0, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}[out]
    return 2 * (n + 1) * 2.0 ** -23 * size + eps * np.abs(x @ w.T) + (2.0 ** -24 if out == "f16" else 2.0 ** -126)


def product(T, N, K, out="f32", seed=0, pad=0, spread=1.0):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    make = lambda r: (torch.randn(r, K, generator=gen, device="cuda") *
                      torch.exp2(torch.randn(r, K, generator=gen, device="cuda") * spread))
    (x, xs, _), (w, ws, _) = quantized(make(T), pad=pad), quantized(make(N), pad=pad)
    flat, y = padded(T, N, 5 * pad, TYPES[out], pad, fill=3)
    dstd.mx4_matmul(x, xs, w, ws, y)
    assert dstd.device_status() == 0
    a, b = decoded(x, xs, K), decoded(w, ws, K)
    off = np.abs(host(y) - a @ b.T)
    assert (off <= bound(a, b, out)).all(), (off / bound(a, b, out)).max()
    mine = torch.zeros_like(flat, dtype=torch.bool)
    mine[pad:pad + T * (N + 5 * pad)].view(T, N + 5 * pad)[:, :N] = True
    assert (flat[~mine] == 3).all()
    return y


@pytest.mark.parametrize("K", [1, 31, 32, 33, 64, 65, 96, 127, 128, 129, 160, 256, 257, 500, 512, 1000, 1025, 4160])
@pytest.mark.parametrize("T,N", [(1, 1), (5, 130), (33, 65)])
def test_product_lengths(T, N, K):
    product(T, N, K, seed=K)


@pytest.mark.parametrize("T", [1, 2, 7, 8, 9, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 255, 256, 257, 300, 513])
@pytest.mark.parametrize("N", [1, 8, 127, 128, 129, 256, 257, 600])
def test_product_sides(T, N):
    product(T, N, 200, seed=T + N)


@pytest.mark.parametrize("out", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("T,N,K", [(1, 257, 300), (37, 801, 1023), (300, 130, 96), (520, 700, 784)])
def test_product_types_and_padded_rows(T, N, K, out):
    product(T, N, K, out, pad=1, spread=0.5 if out == "f16" else 1.0)
    product(T, N, K, out, pad=3, spread=0.5 if out == "f16" else 1.0)


@pytest.mark.parametrize("T,N,K", [(8, 3000, 9000), (1, 4096, 4096), (700, 1500, 5000), (2000, 100, 3000),
                                   (3000, 9, 700), (1024, 1024, 16384)])
def test_product_large(T, N, K):
    product(T, N, K)


@pytest.mark.parametrize("T,N,K,width,parts,exchanged", PLANS)
def test_product_plans(T, N, K, width, parts, exchanged):
    """Every form of the product (mx4_plans.py), fp32 and bf16."""
    product(T, N, K)
    product(T, N, K, "bf16", pad=1)


@pytest.mark.parametrize("out", ["f32", "bf16"])
@pytest.mark.parametrize("T,N,K,pad", [(2100, 2400, 300, 0), (4100, 2500, 97, 1), (2305, 2561, 2049, 0), (20000, 300, 33, 3)])
def test_product_on_pairs(T, N, K, pad, out):
    """Tiles of SM pairs: several to a pair, ragged on both sides, K that ends within a stage."""
    product(T, N, K, out, pad=pad)


def test_product_of_ends():
    """Scales near both ends, zeros, and NaN blocks that reach their own row or channel alone."""
    x = torch.ones(4, 96)
    x[1] *= 1e-38
    x[2] *= 1e36
    x[3, 40] = float("nan")
    w = torch.ones(3, 96)
    w[1] *= 1e-30
    w[2, 0] = float("inf")
    (xq, xs, _), (wq, ws, _) = quantized(x.cuda()), quantized(w.cuda())
    y = torch.empty(4, 3, device="cuda")
    dstd.mx4_matmul(xq, xs, wq, ws, y)
    got, a, b = host(y), decoded(xq, xs, 96), decoded(wq, ws, 96)
    assert np.isnan(got[3]).all() and np.isnan(got[:, 2]).all()
    want = a[:3] @ b[:2].T
    normal = np.abs(want) > 2.0 ** -126
    assert (np.abs(got[:3, :2] - want)[normal] <= 1e-6 * want[normal]).all() and normal.sum() == 5


def test_product_of_nothing():
    e = lambda *s: torch.empty(*s, dtype=torch.uint8, device="cuda")
    y = torch.full((3, 5), 7.0, device="cuda")
    dstd.mx4_matmul(e(3, 0), e(0), e(5, 0), e(0), y)
    assert (y == 0).all()
    y = torch.full((3, 5), 7.0, device="cuda").bfloat16()
    dstd.mx4_matmul(e(3, 0), e(0), e(5, 0), e(0), y)
    assert (y == 0).all()
    dstd.mx4_matmul(e(0, 16), e(0), e(5, 16), e(512), torch.empty(0, 5, device="cuda"))
    dstd.mx4_matmul(e(3, 16), e(512), e(0, 16), e(0), torch.empty(3, 0, device="cuda"))
    torch.cuda.synchronize()


def test_rows_past_the_last_may_hold_anything():
    """Scale bytes of rows past the last are not used: NaN there changes nothing."""
    x, w = torch.randn(5, 300, device="cuda"), torch.randn(140, 300, device="cuda")
    (xq, xs, _), (wq, ws, _) = quantized(x), quantized(w)
    y = torch.empty(5, 140, device="cuda")
    dstd.mx4_matmul(xq, xs, wq, ws, y)
    for s, R in ((xs, 5), (ws, 140)):
        r, b = np.arange(R)[:, None], np.arange(12)[None, :]
        mine = np.zeros(s.numel(), bool)
        mine[mx4.scale_place(r, b, 300)] = True
        s[torch.from_numpy(~mine).cuda()] = 255
    z = torch.empty(5, 140, device="cuda")
    dstd.mx4_matmul(xq, xs, wq, ws, z)
    assert torch.equal(y, z)


def test_product_bits_do_not_change():
    x, w = torch.randn(70, 5000, device="cuda"), torch.randn(300, 5000, device="cuda")
    (xq, xs, _), (wq, ws, _) = quantized(x), quantized(w)
    first = torch.empty(70, 300, device="cuda")
    dstd.mx4_matmul(xq, xs, wq, ws, first)
    for _ in range(5):
        y = torch.empty(70, 300, device="cuda")
        dstd.mx4_matmul(xq, xs, wq, ws, y)
        assert torch.equal(first, y)


def test_streams_and_a_graph():
    """Quantiser and product on a side stream, captured and replayed on new data."""
    x, w = torch.randn(40, 700, device="cuda"), torch.randn(200, 700, device="cuda")
    wq, ws, _ = quantized(w)
    q = torch.empty(40, dstd.mx4_row_bytes(700), dtype=torch.uint8, device="cuda")
    s = torch.empty(dstd.mx4_scale_bytes(40, 700), dtype=torch.uint8, device="cuda")
    y = torch.empty(40, 200, device="cuda")
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        dstd.quantize_mx4(x, q, s)
        dstd.mx4_matmul(q, s, wq, ws, y)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        dstd.quantize_mx4(x, q, s, stream=stream)
        dstd.mx4_matmul(q, s, wq, ws, y, stream=stream)
    for seed in range(3):
        x.copy_(torch.randn(40, 700, generator=torch.Generator().manual_seed(seed)))
        graph.replay()
        torch.cuda.synchronize()
        a, b = mx4.quantize(host(x))[2], decoded(wq, ws, 700)
        assert (np.abs(host(y) - a @ b.T) <= bound(a, b, "f32")).all()


def layer(M, **kw):
    return dstd.params(dict(dict(tau_v=0.5, tau_I=0.25, v_th=1.0, t_first=0.0, t_end=1.2, M=M, t_offset=0.3 / M), **kw), 0.25)


@pytest.mark.parametrize("B,N_in,N_out,M,taus", [(1, 1, 1, 1, (0.5, 0.25)), (3, 50, 70, 10, (0.5, 0.25)),
                                                (16, 256, 300, 32, (0.4, 0.4)), (5, 784, 800, 32, (0.5, 0.25)),
                                                (2, 130, 40, 100, (float("inf"), 0.3)), (4, 33, 129, 128, (0.5, 0.25)),
                                                (64, 300, 2500, 32, (0.5, 0.25)), (1, 64, 5000, 16, (0.5, 0.25))])
def test_layer_forward(B, N_in, N_out, M, taus):
    """The layer on codes gives what its parts give: binning, quantiser, product, scan."""
    gen = torch.Generator(device="cuda").manual_seed(N_in)
    p = layer(M, tau_v=taus[0], tau_I=taus[1], gamma_q=1e-3, gamma_head=0.05, t_head_l=0.3)
    t = torch.rand(B, N_in, generator=gen, device="cuda") * 1.4 - 0.1
    t[torch.rand(B, N_in, generator=gen, device="cuda") < 0.1] = float("inf")
    W = torch.randn(N_out, N_in, generator=gen, device="cuda") / N_in ** 0.5 + 12.0 / N_in
    wq, ws, wv = quantized(W, True)
    wq = wq.contiguous()
    t_out, saved = torch.empty(B, N_out, device="cuda"), torch.empty(dstd.dense_saved_bytes(B, N_out), dtype=torch.uint8, device="cuda")
    pen = torch.empty(4, device="cuda")
    work = torch.full((dstd.dense_mx4_workspace_bytes(B, N_in, N_out, p),), 0xFF, dtype=torch.uint8, device="cuda")
    dstd.dense_fwd_mx4(t, wq, ws, p, t_out, saved, pen, work)
    assert dstd.device_status() == 0
    s = torch.empty(B, M, N_in, device="cuda")
    dstd.binning(t, p, s)
    xq, xs, _ = quantized(s.view(B * M, N_in))
    what = torch.empty(B * M, N_out, device="cuda")
    dstd.mx4_matmul(xq, xs, wq, ws, what)
    a, b = decoded(xq, xs, N_in), decoded(wq, ws, N_in)
    assert (np.abs(host(what) - a @ b.T) <= bound(a, b, "f32")).all()
    want, pen2 = torch.empty(B, N_out, device="cuda"), torch.empty(4, device="cuda")
    dstd.scan_solve(what.view(B, M, N_out).transpose(1, 2).contiguous(), p, wv.sum(1), want, None, pen2)
    # the sums may be formed in another order: a crossing near the threshold may come or go
    same = torch.isfinite(t_out) == torch.isfinite(want)
    assert same.float().mean() >= 0.99
    both = torch.isfinite(t_out) & torch.isfinite(want)
    assert ((t_out - want)[both].abs() <= 1e-4 * 1.2).float().mean() >= 0.99 if both.any() else True
    assert torch.allclose(pen[:2], pen2[:2], rtol=2e-2, atol=1e-6)
    alone, pen3 = torch.empty_like(t_out), torch.empty(4, device="cuda")
    one = torch.empty(dstd.dense_mx4_workspace_bytes(1, N_in, N_out, p), dtype=torch.uint8, device="cuda")
    s1 = torch.empty(dstd.dense_saved_bytes(1, N_out), dtype=torch.uint8, device="cuda")
    for i in range(min(B, 2)):
        t1 = torch.empty(1, N_out, device="cuda")
        dstd.dense_fwd_mx4(t[i:i + 1].clone(), wq, ws, p, t1, s1, pen3, one)
        fine = torch.isfinite(t1[0]) & torch.isfinite(t_out[i])
        assert ((t1[0] - t_out[i])[fine].abs() <= 1e-4 * 1.2).all()


@pytest.mark.parametrize("B,N_in,N_out,M", [(1, 1, 1, 1), (3, 33, 5, 1), (2, 50, 70, 10), (5, 127, 33, 100), (4, 160, 129, 128),
                                            (16, 784, 300, 32), (3, 515, 40, 128), (129, 130, 600, 8)])
def test_layer_forward_step_by_step(B, N_in, N_out, M):
    """What the layer leaves in its workspace: the grid weights' codes and scales are those of quantising the rows that
    the binning gives (zero rows from M up to the padded M), w^ is their product with the weights, and the spikes are
    the scan's of that w^."""
    gen = torch.Generator(device="cuda").manual_seed(M + N_in)
    # weights of 12 in all, nine tenths of them spread over 1.6 s, raise v to 12 0.9 / 1.6 tau_v tau_I = 0.84 at most:
    # with v_th = 0.3 most neurons fire
    p = layer(M, v_th=0.3)
    t = torch.rand(B, N_in, generator=gen, device="cuda") * 1.6 - 0.3        # before the first and behind the last grid point too
    t[torch.rand(B, N_in, generator=gen, device="cuda") < 0.1] = float("inf")
    t[0, :: 7] = -0.3 / M + 1.2 / M * (M // 2)                              # on a grid point, or next to it
    W = torch.randn(N_out, N_in, generator=gen, device="cuda") / N_in ** 0.5 + 12.0 / N_in
    wq, ws, _ = quantized(W)
    t_out = torch.empty(B, N_out, device="cuda")
    saved = torch.empty(dstd.dense_saved_bytes(B, N_out), dtype=torch.uint8, device="cuda")
    work = torch.full((dstd.dense_mx4_workspace_bytes(B, N_in, N_out, p),), 0xFF, dtype=torch.uint8, device="cuda")
    dstd.dense_fwd_mx4(t, wq, ws, p, t_out, saved, None, work)
    assert dstd.device_status() == 0
    Mp = 8
    while Mp < M:
        Mp *= 2
    T, row, up = B * Mp, dstd.mx4_row_bytes(N_in), lambda n: -(-n // 256) * 256
    scale_at = up(4 * N_out)                     # row sums, scales, codes, w^, each from a multiple of 256
    code_at = up(scale_at + dstd.mx4_scale_bytes(T, N_in))
    what_at = up(code_at + T * row)
    assert what_at + 4 * T * N_out == work.numel()
    s = torch.empty(B, M, N_in, device="cuda")
    dstd.binning(t, p, s)
    rows = torch.zeros(B, Mp, N_in, device="cuda")
    rows[:, :M] = s
    want_q, want_s, _ = quantized(rows.view(T, N_in))
    assert torch.equal(work[code_at:code_at + T * row].view(T, row), want_q)
    n = mx4.blocks_of(N_in)
    at = torch.from_numpy(mx4.scale_place(np.arange(T)[:, None], np.arange(-(-n // 4) * 4)[None, :], N_in)).cuda()
    assert torch.equal(work[scale_at:code_at][at], want_s[at])
    what = work[what_at:].view(torch.float32).view(N_out, B, Mp)
    a, b = decoded(want_q, want_s, N_in), decoded(wq, ws, N_in)
    assert (np.abs(host(what.reshape(N_out, T).t()) - a @ b.T) <= bound(a, b, "f32")).all()
    want = torch.empty(B, N_out, device="cuda")
    dstd.scan_solve(what[:, :, :M].permute(1, 0, 2).contiguous(), p, None, want, None, None)
    if M % 4 == 0:                               # the scan's same form
        assert torch.equal(t_out, want)
    assert N_in == 1 or torch.isfinite(t_out).any()

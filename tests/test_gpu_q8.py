"""8-bit rows, their products and the 8-bit layer on the GPU.

What is compared, and how far it may be off:
  codes    within half a code of x 127 / a in 64 bits, plus what two fp32
           roundings move it by (127 * 2^-22); scales to one fp32 rounding;
  values   equal to the fp32 product of code and scale;
  products equal: the sum is a whole number, formed in 64 bits here, and the
           three roundings after it are IEEE (fp32 of the sum, two products),
           then one to 16 bits;
  layer    the spike-time tolerances of the dense tests, on the codes that
           the public quantiser gives.
"""

import math

import numpy as np
import pytest
import torch

from helpers import decode_saved, dense_layer, f32, grid_of, rel_l2, well_conditioned
from oracle import dstd as odstd

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def lib():
    from paper_2607_14672_gb300 import build, dstd
    build.build()
    dstd.load()
    assert dstd.device_status(clear=True) == 0
    yield
    assert dstd.device_status(clear=True) == 0


def padded(a, pad, dtype):
    """A CUDA copy of matrix ``a`` whose rows are ``pad`` elements longer, the rest filled with what must not count."""
    R, K = a.shape
    full = torch.full((R, K + pad), 77, dtype=dtype, device="cuda")
    full[:, :K] = torch.as_tensor(a).to(dtype)
    return full[:, :K]


# ---------------------------------------------------------------------------
# quantiser
# ---------------------------------------------------------------------------
def check_rows(x, q, scale, values):
    """x: float64 array of what the GPU saw."""
    a = np.abs(x).max(axis=1, initial=0.0)
    finite = np.isfinite(x).all(axis=1)
    ratio = np.divide(x, a[:, None], out=np.zeros_like(x), where=(a[:, None] > 0) & finite[:, None]) * 127.0
    off = np.abs(q - ratio)[finite]
    assert off.size == 0 or off.max() <= 0.5 + 127 * 2.0 ** -22
    assert np.abs(q).max(initial=0) <= 127
    ref = (a / 127.0)[finite]
    # one rounding of the scale: relative, or half the smallest subnormal
    assert np.all(np.abs(scale[finite] - ref) <= np.maximum(ref * 2.0 ** -24, 2.0 ** -150) * (1 + 1e-12))
    assert np.isnan(scale[~finite]).all() and (q[~finite] == 0).all()
    want = q.astype(np.float32) * scale.astype(np.float32)[:, None]
    np.testing.assert_array_equal(values.astype(np.float32), want)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("R,K,pad", [(1, 1, 0), (3, 7, 0), (5, 64, 3), (2, 255, 1), (4, 256, 0), (7, 1023, 9),
                                     (3, 4096, 4), (2, 16384, 0), (1, 16385, 0), (2, 40000, 0), (300, 33, 0)])
def test_quantize_rows(dtype, R, K, pad):
    from paper_2607_14672_gb300 import dstd
    g = np.random.default_rng(R * 1000 + K)
    x = padded(g.normal(size=(R, K)) * 10.0 ** g.integers(-3, 3, (R, 1)), pad, dtype)
    q = padded(np.zeros((R, K)), pad, torch.int8)
    values = padded(np.zeros((R, K)), pad, torch.float32)
    scale = torch.empty(R, device="cuda")
    dstd.quantize_rows(x, q, scale, values)
    q2 = torch.empty(R, K, dtype=torch.int8, device="cuda")
    scale2 = torch.empty(R, device="cuda")
    dstd.quantize_rows(x, q2, scale2)
    torch.cuda.synchronize()
    check_rows(x.double().cpu().numpy(), q.cpu().numpy().astype(int), scale.cpu().numpy(), values.cpu().numpy())
    assert torch.equal(q, q2) and torch.equal(scale, scale2)
    if pad and R > 1:  # what lies between the rows stays
        assert (q.as_strided((R - 1, pad), (K + pad, 1), q.storage_offset() + K) == 77).all()
        assert (values.as_strided((R - 1, pad), (K + pad, 1), K) == 77).all()


def test_quantize_rows_extremes():
    """Zeros, subnormals, the largest values, ties, infinities and NaN."""
    from paper_2607_14672_gb300 import dstd
    K = 37
    rows = [np.zeros(K), -np.zeros(K), np.full(K, 1e-45), np.full(K, -3e-42), np.linspace(-1e-38, 1e-38, K),
            np.linspace(-2e-30, 1e-30, K), np.linspace(-3.4e38, 3.4e38, K), np.r_[127.0, np.arange(36) + 0.5],
            np.r_[np.inf, np.ones(K - 1)], np.r_[np.ones(K - 1), -np.inf], np.r_[1.0, np.nan, np.ones(K - 2)],
            np.r_[np.nan, np.inf, np.zeros(K - 2)]]
    x = torch.tensor(np.array(rows), dtype=torch.float32, device="cuda")
    q = torch.empty(x.shape, dtype=torch.int8, device="cuda")
    scale, values = torch.empty(len(rows), device="cuda"), torch.empty(x.shape, device="cuda")
    dstd.quantize_rows(x, q, scale, values)
    check_rows(x.double().cpu().numpy(), q.cpu().numpy().astype(int), scale.cpu().numpy(), values.cpu().numpy())
    assert q[7].tolist() == [127] + [int(np.rint(v)) for v in np.arange(36) + 0.5]   # ties to even
    # no rows, no columns
    dstd.quantize_rows(x[:0], q[:0], scale[:0])
    dstd.quantize_rows(x[:, :0], q[:, :0], scale, values[:, :0])
    torch.cuda.synchronize()
    assert (scale == 0).all()


# ---------------------------------------------------------------------------
# product
# ---------------------------------------------------------------------------
def product(x, sx, w, sw, out):
    from paper_2607_14672_gb300 import dstd
    T, K = x.shape
    ws = torch.full((dstd.int8_matmul_workspace_bytes(T, w.shape[0], K),), 255, dtype=torch.uint8, device="cuda")
    dstd.int8_matmul(x, sx, w, sw, out, ws)
    torch.cuda.synchronize()
    assert dstd.device_status() == 0


def expected(x, sx, w, sw, dtype):
    """The product from 64-bit whole sums (fp64 holds them exactly below 2^53)."""
    sums = (x.double() @ w.double().t()).to(torch.int64) if x.shape[1] else torch.zeros(
        x.shape[0], w.shape[0], dtype=torch.int64, device=x.device)
    return ((sums.double().float() * sx[:, None]) * sw[None, :]).to(dtype)


def random_case(T, N, K, pad, seed, dtype=torch.float32):
    g = torch.Generator(device="cuda").manual_seed(seed)
    code = lambda R: torch.randint(-128, 128, (R, K), generator=g, device="cuda")
    x, w = padded(code(T), pad, torch.int8), padded(code(N), pad, torch.int8)
    sx = torch.rand(T, generator=g, device="cuda") + 0.01
    sw = torch.rand(N, generator=g, device="cuda") * 0.01 + 1e-5
    out = padded(torch.zeros(T, N), pad, dtype)
    return x, sx, w, sw, out


SHAPES = [(1, 1, 1, 0), (1, 5, 16, 0), (2, 3, 15, 0), (3, 130, 17, 0), (1, 4096, 4096, 0), (4, 100, 1000, 1),
          (7, 33, 4097, 0), (8, 300, 2048, 16), (9, 257, 784, 0), (15, 64, 129, 7), (16, 255, 1024, 0),
          (17, 300, 1040, 0), (31, 801, 1023, 9), (32, 256, 2064, 0), (33, 512, 64, 0), (64, 1000, 1100, 4),
          (65, 10, 784, 0), (100, 300, 5000, 0), (128, 128, 128, 16), (129, 1025, 48, 0), (192, 256, 1200, 0),
          (200, 513, 2050, 0), (256, 800, 784, 0), (385, 700, 3000, 3), (1000, 1000, 1000, 0), (1500, 260, 16, 0),
          (2500, 40, 333, 0), (3000, 3100, 96, 0), (7000, 20, 1000, 0), (5000, 8, 300, 0), (9000, 1, 4100, 0),
          (3000, 100, 2000, 0), (2000, 33, 64, 5), (9000, 150, 500, 7), (4000, 129, 1040, 0), (20000, 64, 2048, 0)]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("T,N,K,pad", SHAPES)
def test_int8_matmul(T, N, K, pad, dtype):
    x, sx, w, sw, out = random_case(T, N, K, pad, T * 7 + N * 3 + K, dtype)
    product(x, sx, w, sw, out)
    want = expected(x, sx, w, sw, dtype)
    assert torch.equal(out, want), (out.float() - want.float()).abs().max().item()
    if pad and T > 1:
        assert (out.as_strided((T - 1, pad), (N + pad, 1), N) == 77).all()


@pytest.mark.parametrize("T", [1, 6, 24, 200])
@pytest.mark.parametrize("K", [1024, 1040, 5000, 131071])
def test_int8_matmul_sums_are_exact(T, K):
    """Rows whose partial sums pass 2^24 (fp32 could not hold them) and come near 2^31."""
    g = torch.Generator(device="cuda").manual_seed(K + T)
    N = 300
    x = torch.full((T, K), -128, dtype=torch.int8, device="cuda")
    w = torch.full((N, K), -128, dtype=torch.int8, device="cuda")
    for m in (x, w):
        m[1:] = torch.randint(101, 128, m[1:].shape, generator=g, device="cuda")
    w[N // 2:] *= -1
    one = lambda n: torch.ones(n, device="cuda")
    out = torch.empty(T, N, device="cuda")
    product(x, one(T), w, one(N), out)
    assert torch.equal(out, expected(x, one(T), w, one(N), torch.float32))
    assert out[0, 0].item() == np.float32(16384.0 * K)


@pytest.mark.parametrize("T", [3, 40])
def test_int8_matmul_misaligned(T):
    """Rows that start at odd addresses, with strides that are no multiple of 16."""
    N, K = 150, 777
    g = torch.Generator(device="cuda").manual_seed(5)
    for off in (1, 2, 3, 8, 13):
        buf = torch.randint(-128, 128, ((T + N) * (K + 3) + 64,), generator=g, device="cuda").to(torch.int8)
        x = buf[off:].as_strided((T, K), (K + 3, 1), off)
        w = buf[off:].as_strided((N, K), (K + 2, 1), off + T * (K + 3))
        sx, sw = torch.rand(T, device="cuda"), torch.rand(N, device="cuda")
        out = torch.empty(T * N + 1, device="cuda")[1:].view(T, N)
        product(x, sx, w, sw, out)
        assert torch.equal(out, expected(x, sx, w, sw, torch.float32))


@pytest.mark.parametrize("T,N,K", [(40, 3000, 4096), (9000, 64, 1024), (600, 600, 784), (5, 100, 64)])
def test_aligned_workspace(T, N, K):
    """The smaller workspace serves aligned operands, and is refused for others."""
    from paper_2607_14672_gb300 import dstd
    x, sx, w, sw, out = random_case(T, N, K, 0, 31)
    small, full = (dstd.int8_matmul_workspace_bytes(T, N, K, aligned=a) for a in (True, False))
    assert small <= full and (small < full or T < 9)
    room = torch.full((small + 256,), 85, dtype=torch.uint8, device="cuda")
    dstd.int8_matmul(x, sx, w, sw, out, room[:small])
    torch.cuda.synchronize()
    assert torch.equal(out, expected(x, sx, w, sw, torch.float32)) and (room[small:] == 85).all()
    if T >= 9:
        for which in range(2):  # either operand's rows at other addresses
            y = padded((x if which else w).cpu(), 1, torch.int8)
            with pytest.raises(dstd.DstdError) as e:
                dstd.int8_matmul(y if which else x, sx, w if which else y, sw, out, room[:small])
            assert e.value.code == -3


def test_int8_matmul_empty():
    for T, N, K in ((0, 5, 16), (5, 0, 16), (5, 7, 0), (40, 70, 0)):
        x, w = torch.zeros(T, K, dtype=torch.int8, device="cuda"), torch.zeros(N, K, dtype=torch.int8, device="cuda")
        out = torch.full((T, N), 3.0, device="cuda")
        product(x, torch.ones(T, device="cuda"), w, torch.ones(N, device="cuda"), out)
        assert (out == 0).all()


@pytest.mark.parametrize("T", [2, 50])
def test_int8_matmul_scales_that_are_not_finite(T):
    """A token whose row was not finite gives NaN in its row alone."""
    x, sx, w, sw, out = random_case(T, 40, 128, 0, 3)
    sx[1] = math.nan
    sw[7] = math.inf
    product(x, sx, w, sw, out)
    want = expected(x, sx, w, sw, torch.float32)
    assert torch.equal(out.nan_to_num(1e30), want.nan_to_num(1e30))
    assert out[1].isnan().all() and not out[0, :7].isnan().any()


def test_int8_matmul_past_32_bit_offsets():
    """Weights and outputs whose offsets pass 2^31 elements (2.2 GB of codes)."""
    N, K, T = 270000, 8192, 2
    w = torch.empty(N, K, dtype=torch.int8, device="cuda")
    w.random_(-128, 128)
    x = torch.randint(-128, 128, (T, K), device="cuda").to(torch.int8)
    sx, sw = torch.rand(T, device="cuda"), torch.rand(N, device="cuda")
    out = torch.empty(T, N, device="cuda")
    product(x, sx, w, sw, out)
    at = torch.tensor([0, 1, N // 2, 262143, 262144, 262145, N - 1], device="cuda")
    assert torch.equal(out[:, at], expected(x, sx, w[at], sw[at], torch.float32))
    # 40 tokens of a buffer with rows 2^27 apart: token and output offsets pass 2^32
    del w
    T, N, K, ld = 40, 64, 48, 1 << 27
    xs = torch.empty(39 * ld + K, dtype=torch.int8, device="cuda")
    x = xs.as_strided((T, K), (ld, 1))
    x.copy_(torch.randint(-128, 128, (T, K), device="cuda"))
    w = torch.randint(-128, 128, (N, K), device="cuda").to(torch.int8)
    sx, sw = torch.rand(T, device="cuda"), torch.rand(N, device="cuda")
    out = torch.empty(39 * ld + N, dtype=torch.bfloat16, device="cuda").as_strided((T, N), (ld, 1))
    product(x, sx, w, sw, out)
    assert torch.equal(out, expected(x, sx, w, sw, torch.bfloat16))


def test_int8_matmul_streams_and_graph():
    """On a stream of its own, and captured in a graph that is replayed on new codes."""
    from paper_2607_14672_gb300 import dstd
    for T in (2, 80):
        x, sx, w, sw, out = random_case(T, 300, 1100, 0, 11)
        ws = torch.empty(dstd.int8_matmul_workspace_bytes(T, 300, 1100), dtype=torch.uint8, device="cuda")
        s = torch.cuda.Stream()
        s.wait_stream(torch.cuda.current_stream())
        dstd.int8_matmul(x, sx, w, sw, out, ws, stream=s)
        s.synchronize()
        assert torch.equal(out, expected(x, sx, w, sw, torch.float32))
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            dstd.int8_matmul(x, sx, w, sw, out, ws, stream=s)
        for seed in (1, 2):
            x.copy_(random_case(T, 300, 1100, 0, seed)[0])
            out.zero_()
            torch.cuda.synchronize()
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(out, expected(x, sx, w, sw, torch.float32))


@pytest.mark.parametrize("T,N,K", [(3, 1000, 2048), (150, 1000, 2048)])
def test_capture_after_copies_and_joins(T, N, K):
    """Captured behind a copy, behind a fill on a forked stream and in a row of its own kind: replays see the new inputs."""
    from paper_2607_14672_gb300 import dstd
    src, sx, w, sw, out = random_case(T, N, K, 0, 21)
    x, out2, half = torch.zeros_like(src), torch.empty_like(out), torch.empty(T, N, dtype=torch.bfloat16, device="cuda")
    scratch = torch.empty(dstd.int8_matmul_workspace_bytes(T, N, K), dtype=torch.uint8, device="cuda")
    dstd.int8_matmul(x, sx, w, sw, out, scratch)
    torch.cuda.synchronize()
    s, side = torch.cuda.Stream(), torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        x.copy_(src)
        dstd.int8_matmul(x, sx, w, sw, out, scratch, stream=s)
        side.wait_stream(s)
        with torch.cuda.stream(side):
            half.fill_(1.0)
        s.wait_stream(side)
        dstd.int8_matmul(x, sx, w, sw, half, scratch, stream=s)
        dstd.int8_matmul(x, sx, w, sw, out2, scratch, stream=s)
    for seed in (3, 4):
        src.copy_(random_case(T, N, K, 0, seed)[0])
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        want = expected(src, sx, w, sw, torch.float32)
        assert torch.equal(out, want) and torch.equal(out2, want) and torch.equal(half, want.bfloat16())


@pytest.mark.parametrize("T,N,K", [(3, 3000, 4096), (70, 3000, 4096), (300, 2000, 1500)])
def test_codes_written_just_before_the_product(T, N, K):
    """Weights and tokens quantised right before the product on the same stream,
    again and again: what the quantiser writes is what the product reads."""
    from paper_2607_14672_gb300 import dstd
    g = torch.Generator(device="cuda").manual_seed(T)
    w = [torch.randn(N, K, generator=g, device="cuda") for _ in range(2)]
    x = [torch.randn(T, K, generator=g, device="cuda") for _ in range(2)]
    wq, xq = torch.empty(N, K, dtype=torch.int8, device="cuda"), torch.empty(T, K, dtype=torch.int8, device="cuda")
    ws, xs = torch.empty(N, device="cuda"), torch.empty(T, device="cuda")
    scratch = torch.empty(dstd.int8_matmul_workspace_bytes(T, N, K), dtype=torch.uint8, device="cuda")
    outs = [torch.empty(T, N, device="cuda") for _ in range(12)]
    for i, o in enumerate(outs):
        dstd.quantize_rows(x[i % 2], xq, xs)
        dstd.quantize_rows(w[i % 2], wq, ws)
        dstd.int8_matmul(xq, xs, wq, ws, o, scratch)
    torch.cuda.synchronize()
    for k in range(2):
        dstd.quantize_rows(x[k], xq, xs)
        dstd.quantize_rows(w[k], wq, ws)
        torch.cuda.synchronize()
        want = expected(xq, xs, wq, ws, torch.float32)
        assert all(torch.equal(o, want) for o in outs[k::2])


# ---------------------------------------------------------------------------
# layer
# ---------------------------------------------------------------------------
def run_q8(t_in, layer, norm):
    from paper_2607_14672_gb300 import dstd
    B, N_in = t_in.shape
    N_out = layer["W"].shape[0]
    dev = lambda a: torch.tensor(np.asarray(a), dtype=torch.float32, device="cuda")
    p = dstd.params(layer, norm)
    W = dev(layer["W"])
    wq, ws_, Wv = torch.empty(W.shape, dtype=torch.int8, device="cuda"), torch.empty(N_out, device="cuda"), dev(W.cpu())
    dstd.quantize_rows(W, wq, ws_, Wv)
    scratch = torch.empty(dstd.dense_q8_workspace_bytes(B, N_in, N_out, p), dtype=torch.uint8, device="cuda")
    t_out = torch.empty(B, N_out, device="cuda")
    saved = torch.empty(dstd.dense_saved_bytes(B, N_out), dtype=torch.uint8, device="cuda")
    pen = torch.empty(4, device="cuda")
    t = dev(t_in)
    dstd.dense_fwd_q8(t, wq, ws_, p, t_out, saved, pen, scratch)
    torch.cuda.synchronize()
    return p, t, wq, ws_, Wv, t_out, saved, pen


@pytest.mark.parametrize("B,N_in,N_out,M", [(1, 64, 32, 16), (3, 37, 130, 20), (8, 200, 300, 32), (16, 784, 100, 8),
                                            (2, 1500, 257, 64), (1, 5, 1, 1), (5, 333, 70, 128)])
def test_dense_fwd_q8(B, N_in, N_out, M):
    from paper_2607_14672_gb300 import dstd
    t_in, layer = dense_layer(B, N_in, N_out, M, 0.5, 0.25, seed=N_in, t_offset=0.0, gammas=(0.05, 0.01, 1e-3))
    t_in = f32(t_in)
    t_in[0] = np.inf                                   # a sample without a spike: tokens of zeros
    layer["W"] = f32(layer["W"])
    p, t, wq, w_scale, Wv, t_out, saved, pen = run_q8(t_in, layer, 1.0 / B)
    # the tokens' codes, as the public binning and quantiser give them
    s = torch.empty(B, M, N_in, device="cuda")
    dstd.binning(t, p, s)
    q = torch.empty(B * M, N_in, dtype=torch.int8, device="cuda")
    scale = torch.empty(B * M, device="cuda")
    dstd.quantize_rows(s.view(B * M, N_in), q, scale)
    sums = (q.double() @ wq.double().t()) * scale.double()[:, None] * w_scale.double()[None, :]
    what = sums.view(B, M, N_out).permute(0, 2, 1).cpu().numpy()
    T, dt = grid_of(layer)
    ctx = odstd.solve(what, T, dt, 0.5, 0.25, 1.0)
    tg = t_out.cpu().numpy().astype(np.float64)
    ok = well_conditioned(ctx, 1.0)
    fired = np.isfinite(ctx["t"])
    assert np.array_equal(fired[ok], np.isfinite(tg)[ok])
    both = ok & fired
    assert both.sum() == 0 or np.abs(tg[both] - ctx["t"][both]).max() <= 1e-4 * 1.2
    if B > 1 and N_in > 30:
        assert both.any()
    assert np.isinf(tg[0]).all()
    counts = pen.cpu().numpy()
    assert counts[2] == np.isinf(tg).sum() and counts[3] == np.isfinite(tg).sum()
    # the dead-neuron penalty: gamma_q norm sum over silent (b, i) of sum_j (0 - w_ij), as in the fp32 layer
    silent = np.isinf(tg).sum(axis=0)
    rowsum = w_scale.cpu().numpy().astype(np.float64) * wq.cpu().numpy().astype(np.float64).sum(axis=1)
    assert counts[1] == pytest.approx(-1e-3 / B * (silent * rowsum).sum(), rel=1e-4, abs=1e-9)


def test_dense_fwd_q8_without_penalty():
    """No penalty asked for, or one without the dead-neuron term: the same times, and that term is 0."""
    from paper_2607_14672_gb300 import dstd
    B, N_in, N_out, M = 3, 120, 90, 16
    t_in, layer = dense_layer(B, N_in, N_out, M, 0.5, 0.25, seed=8, gammas=(0.05, 0.01, 0.0))
    t_in, layer["W"] = f32(t_in), f32(layer["W"])
    p, t, wq, w_scale, _, t_out, saved, pen = run_q8(t_in, layer, 1.0 / B)
    assert pen[1].item() == 0 and pen[2].item() + pen[3].item() == B * N_out
    again = torch.empty_like(t_out)
    ws = torch.empty(dstd.dense_q8_workspace_bytes(B, N_in, N_out, p), dtype=torch.uint8, device="cuda")
    dstd.dense_fwd_q8(t, wq, w_scale, p, again, saved, None, ws)
    torch.cuda.synchronize()
    assert torch.equal(again, t_out)


def test_dense_q8_gradient_passes_straight_through():
    """dense_bwd at the weights' values and the 8-bit forward's spike state,
    against the oracle's backward there."""
    from paper_2607_14672_gb300 import dstd
    B, N_in, N_out, M = 6, 200, 300, 32
    t_in, layer = dense_layer(B, N_in, N_out, M, 0.5, 0.25, seed=4, t_offset=0.0)
    t_in, layer["W"] = f32(t_in), f32(layer["W"])
    p, t, wq, w_scale, Wv, t_out, saved, _ = run_q8(t_in, layer, 1.0 / B)
    g = torch.rand(B, N_out, device="cuda")
    g_t, g_W = torch.empty(B, N_in, device="cuda"), torch.empty(N_out, N_in, device="cuda")
    ws = torch.empty(dstd.dense_workspace_bytes(B, N_in, N_out, p, "x3"), dtype=torch.uint8, device="cuda")
    dstd.dense_bwd(t, Wv, t_out, saved, g, p, "x3", g_t, g_W, ws)
    torch.cuda.synchronize()
    q, _, vdot = decode_saved(saved.cpu().numpy(), B, N_out)
    tg = t_out.cpu().numpy().astype(np.float64)
    T, dt = grid_of(layer)
    ctx = dict(t=tg, q=q.astype(int), vdot=vdot.astype(np.float64), fired=np.isfinite(tg),
               s=odstd.binning(t_in, T, dt, 0.5, 0.25))
    gW, gt, _ = odstd.backward_dense(ctx, t_in, Wv.cpu().numpy().astype(np.float64), g.cpu().numpy() * np.isfinite(tg),
                                     T, dt, 0.5, 0.25, 1.0)
    assert rel_l2(g_W.cpu().numpy(), gW) <= 1e-3
    assert rel_l2(g_t.cpu().numpy(), gt) <= 1e-3


def test_network_trains_and_serves_in_8_bits():
    """A q8 network: clipped steps lower the loss, a captured step replays as
    the eager one, and serving on the kept codes gives the forward's times."""
    from paper_2607_14672_gb300 import configs, net
    cfg = configs.config2(batch=32, M=16)
    n = net.DenseNet(cfg, "q8", with_adamw=True, max_norm=0.5)
    n.set_inputs(cfg["inputs"](B=32), cfg["labels"](B=32))
    first = None
    for _ in range(17):
        n.step()
        torch.cuda.synchronize()
        first = n.loss[0].item() if first is None else first
        assert math.isfinite(n.grad_norm.item()) and n.grad_norm.item() > 0
    assert n.loss[0].item() < first
    assert n.adam_state.tolist()[0] == 17
    n.forward()
    times = [t.clone() for t in n.t]
    before = [w.clone() for w in n.W]
    for w in n.W:
        w.fill_(math.nan)                              # serving reads the codes alone
    for t in n.t:
        t.zero_()
    n.serve()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(times, n.t))
    for w, b in zip(n.W, before):
        w.copy_(b)
    # a captured step
    state = [x.clone() for x in n.W + n.m + n.v + [n.adam_state]]
    n.step()
    torch.cuda.synchronize()
    after = [x.clone() for x in n.W + n.m + n.v + [n.adam_state]]
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        n.step(stream=s)
    for x, b in zip(n.W + n.m + n.v + [n.adam_state], state):
        x.copy_(b)
    torch.cuda.synchronize()
    graph.replay()
    torch.cuda.synchronize()
    # the loss and dW sums use fp32 atomics whose order may change the last bits
    for x, b in zip(n.W + n.m + n.v, after[:-1]):
        assert rel_l2(x.cpu().numpy(), b.cpu().numpy()) <= 1e-3
    assert torch.equal(n.adam_state, after[-1])


def test_example_trains_and_serves():
    """The example: a captured training loop, then single samples from the codes
    alone with the batch's spike times (whole-number sums do not depend on the
    number of tokens, nor the scan on the batch)."""
    import importlib.util
    import os
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "q8_mlp.py")
    spec = importlib.util.spec_from_file_location("q8_mlp", path)
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    losses, same = m.main(["--steps", "6", "--batch", "16"])
    assert all(math.isfinite(x) for x in losses) and same

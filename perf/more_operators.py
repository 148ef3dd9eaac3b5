"""Workloads of the operators of 4-bit training and of learning from a teacher: rows
quantised to 4-bit floating point with a power of two for each block of 32, products
of such rows, the largest logits of each row (a teacher's record), and the distillation
loss from such a record with its gradient.

A case is a dict of plain values; ``listed`` gives the named ones, ``draw``
more of the same ranges. ``run`` is one pass: with ``own`` through the
framework's entry points, otherwise in elementary torch operations.
"""

import math

import torch

own = False

DEV = "cuda"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
BYTES = {"f32": 4, "bf16": 2, "f16": 2}
BLOCK = 32                       # columns that share a power of two
TAU_SOFT, T_END = 0.02, 1.2      # of the networks' readout: logits are -t / TAU_SOFT, silent outputs count as T_END
MAGNITUDES = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def listed():
    return [
        # the MLP's first layer before a training step's forward: the values that its 4-bit codes stand for
        dict(name="quantize mlp weights", op="quantize", rows=800, cols=784, type="f32", pad=0),
        # the largest dense layer's weights
        dict(name="quantize 16k weights", op="quantize", rows=16384, cols=16384, type="f32", pad=0),
        # the smallest product: one token through one layer, where latency counts
        dict(name="product 1 token", op="product", tokens=1, cols=4096, rows=4096, x="codes", out="f32", pad=0),
        # one sample of 8 grid points through the largest dense layer, where reading the weights counts
        dict(name="product 8 tokens 16k", op="product", tokens=8, cols=16384, rows=16384, x="codes", out="bf16", pad=0),
        # odd sizes and padded rows: one sample of 37 grid points, activations quantised on the way
        dict(name="product odd", op="product", tokens=37, cols=1023, rows=801, x="f32", out="f32", pad=9),
        # the MLP's first layer on its training batch: 256 samples of 32 grid points
        dict(name="product mlp batch", op="product", tokens=8192, cols=784, rows=800, x="f32", out="f32", pad=0),
        # the largest dense layer: 128 samples of 32 grid points
        dict(name="product 16k batch", op="product", tokens=4096, cols=16384, rows=16384, x="bf16", out="f32", pad=0),
        # the record of a teacher with a 10-class readout: spike times, one in ten silent
        dict(name="top of a readout", op="top", rows=256, cols=10, top=4, type="f32", pad=0, times=True),
        # of a teacher with many classes, 16-bit logits with many ties
        dict(name="top of 32k classes", op="top", rows=4096, cols=32768, top=64, type="bf16", pad=0, times=False),
        # a training step's loss on a 10-class readout, spike times
        dict(name="distill a readout", op="distill", rows=256, cols=10, top=4, type="f32", pad=0, times=True),
        # few long rows, odd and padded
        dict(name="distill few long rows", op="distill", rows=7, cols=131071, top=128, type="f32", pad=3, times=False),
        # many classes in 16 bits
        dict(name="distill 32k classes", op="distill", rows=4096, cols=32768, top=64, type="bf16", pad=0, times=False),
    ]


def _spread(rng, low, high):
    """A whole number of [low, high], spread over its logarithm."""
    return min(high, max(low, int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))))


def draw(rng):
    op = rng.choice(["quantize", "product", "product", "product", "top", "distill"])
    pad = rng.choice([0, 0, rng.randint(1, 17)])
    if op == "quantize":
        return dict(op=op, rows=_spread(rng, 1, 16384), cols=_spread(rng, 8, 16384),
                    type=rng.choice(["f32", "bf16", "f16"]), pad=pad)
    if op == "product":
        cols, rows = _spread(rng, 16, 16384), _spread(rng, 8, 16384)
        tokens = _spread(rng, 1, 16384)
        tokens = max(1, min(tokens, 4096 * 16384 * 16384 // (cols * rows), (1 << 27) // rows, (1 << 27) // cols))
        return dict(op=op, tokens=tokens, cols=cols, rows=rows, x=rng.choice(["codes", "f32", "bf16"]),
                    out=rng.choice(["f32", "bf16"]), pad=pad)
    cols = _spread(rng, 2, 131072)
    rows = max(1, min(_spread(rng, 1, 16384), (1 << 27) // cols))
    return dict(op=op, rows=rows, cols=cols, top=min(cols, _spread(rng, 1, 256)),
                type=rng.choice(["f32", "bf16", "f16"]), pad=pad, times=rng.random() < 0.3)


# -- 4-bit rows ------------------------------------------------------------
# A row of codes: 16 bytes for each block of 32 columns, the even column in a byte's
# low half; columns beyond the end are zero. Exponents (plus 127) in tiles of 128 rows
# by 4 blocks: byte (r % 32) * 16 + (r % 128 / 32) * 4 + b % 4 of a tile's 512.
def _exponents(x):
    """The least e with max |x| <= 6 2^e of each block, at least -127, and the blocks."""
    rows, cols = x.shape
    blocks = (cols + BLOCK - 1) // BLOCK
    x = torch.nn.functional.pad(x, (0, blocks * BLOCK - cols)).reshape(rows, blocks, BLOCK)
    mantissa, e = torch.frexp(x.abs().amax(2))
    e = torch.where(mantissa > 0.75, e - 2, e - 3)
    return torch.where(mantissa == 0, torch.full_like(e, -127), e).clamp_(min=-127), x


def _power(e):
    """2^e as fp32, e of [-127, 127]."""
    normal = ((e + 127).clamp(min=1) << 23).view(torch.float32)
    return torch.where(e < -126, normal * 0.5, normal)


def _magnitudes(x):
    """|x| <= 6 rounded to the values of a code, ties to the even code."""
    step = torch.where(x < 2.0, 0.5, torch.where(x < 4.0, 1.0, 2.0))
    return torch.round(x / step) * step


def _rounded(x):
    """fp32 rows as the values that their codes stand for: signed magnitudes in blocks, and exponents."""
    e, blocks = _exponents(x)
    m = _magnitudes(blocks.abs().mul_(_power(-e)[:, :, None]))
    return torch.where(blocks < 0, -m, m), e


def _values(x):
    m, e = _rounded(x)
    return (m * _power(e)[:, :, None]).reshape(x.shape[0], -1)[:, :x.shape[1]]


def _tiled(e):
    """Exponents [rows, blocks] as bytes in tiles."""
    rows, blocks = e.shape
    e = torch.nn.functional.pad(e + 127, (0, -blocks % 4, 0, -rows % 128)).to(torch.uint8)
    return e.reshape(e.shape[0] // 128, 4, 32, e.shape[1] // 4, 4).permute(0, 3, 2, 1, 4).reshape(-1)


def _packed(x):
    """Codes and exponents of fp32 rows, to make inputs with."""
    m, e = _rounded(x)
    edges = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0], device=x.device)
    code = torch.bucketize(m.abs(), edges).to(torch.uint8) | (m < 0).to(torch.uint8) << 3
    code = code.reshape(x.shape[0], -1)
    return code[:, 0::2] | code[:, 1::2] << 4, _tiled(e)


def _unpacked(q, scale, cols):
    """The values of codes and exponents, as fp32."""
    rows, bytes_ = q.shape
    blocks = bytes_ // 16
    table = torch.tensor(MAGNITUDES + tuple(-v for v in MAGNITUDES), device=q.device)
    low = table.index_select(0, (q & 15).int().reshape(-1)).reshape(rows, bytes_)
    high = table.index_select(0, (q >> 4).int().reshape(-1)).reshape(rows, bytes_)
    v = torch.stack((low, high), 2).reshape(rows, blocks, BLOCK)
    tiles = scale.reshape((rows + 127) // 128, (blocks + 3) // 4, 32, 4, 4).permute(0, 3, 2, 1, 4)
    e = tiles.reshape(tiles.shape[0] * 128, -1)[:rows, :blocks].int() - 127
    return (v * _power(e)[:, :, None]).reshape(rows, -1)[:, :cols]


# -- inputs ----------------------------------------------------------------
def _generator(seed):
    return torch.Generator(device=DEV).manual_seed(int(seed))


def _padded(rows, cols, pad, dtype):
    return torch.empty(rows, cols + pad, dtype=dtype, device=DEV)[:, :cols]


def _weights(rows, cols, gen):
    """W = mu + N(0, 1/fan_in) with mu fan_in = 12, as the dense layers are initialised."""
    return torch.randn(rows, cols, device=DEV, generator=gen).mul_(1.0 / math.sqrt(cols)).add_(12.0 / cols)


def _grid_weights(tokens, cols, gen):
    """Activations of a layer: most inputs carry no weight at a given grid point."""
    x = torch.rand(tokens, cols, device=DEV, generator=gen)
    return x.mul_(torch.rand(tokens, cols, device=DEV, generator=gen) < 0.2)


def _outputs(case, gen):
    """A readout's spike times, one in ten silent, or logits, one in fifty masked."""
    shape = (case["rows"], case["cols"])
    y = _padded(*shape, case["pad"], TYPES[case["type"]])
    if case["times"]:
        t = torch.rand(*shape, device=DEV, generator=gen).mul_(0.2).add_(0.8)
        y.copy_(t.masked_fill_(torch.rand(*shape, device=DEV, generator=gen) < 0.1, math.inf))
    else:
        z = torch.randn(*shape, device=DEV, generator=gen).mul_(2.5)
        y.copy_(z.masked_fill_(torch.rand(*shape, device=DEV, generator=gen) < 0.02, -math.inf))
    return y


def _logits(s, y):
    """fp32 (or 64-bit) logits of outputs, and which of them are silent or masked."""
    z = y * s["factor"]
    none = z == -math.inf
    return (z.masked_fill(none, s["factor"] * T_END) if s["times"] else z), none


def prepare(case, seed):
    gen = _generator(seed)
    s = dict(case)
    if case["op"] == "quantize":
        rows, cols = case["rows"], case["cols"]
        x = _padded(rows, cols, case["pad"], TYPES[case["type"]])
        x.copy_(_weights(rows, cols, gen))
        blocks = (cols + BLOCK - 1) // BLOCK
        s.update(x=x, q=torch.empty(rows, 16 * blocks, dtype=torch.uint8, device=DEV),
                 scale=torch.empty((rows + 127) // 128 * ((blocks + 3) // 4) * 512, dtype=torch.uint8, device=DEV),
                 values=torch.empty(rows, cols, device=DEV))
        return s
    if case["op"] == "product":
        tokens, rows, cols, pad = case["tokens"], case["rows"], case["cols"], case["pad"]
        blocks = (cols + BLOCK - 1) // BLOCK
        codes, s["w_scale"] = _packed(_weights(rows, cols, gen))
        s["w"] = _padded(rows, 16 * blocks, 16 * (pad % 3), torch.uint8)
        s["w"].copy_(codes)
        x = _grid_weights(tokens, cols, gen)
        if case["x"] == "codes":
            codes, s["x_scale"] = _packed(x)
            s["x_in"] = _padded(tokens, 16 * blocks, 16 * (pad % 3), torch.uint8)
            s["x_in"].copy_(codes)
        else:
            s["x_in"] = _padded(tokens, cols, pad, TYPES[case["x"]])
            s["x_in"].copy_(x)
            s["q"] = torch.empty(tokens, 16 * blocks, dtype=torch.uint8, device=DEV)
            s["x_scale"] = torch.empty((tokens + 127) // 128 * ((blocks + 3) // 4) * 512, dtype=torch.uint8, device=DEV)
        s["out_buffer"] = torch.empty(tokens, rows, dtype=TYPES[case["out"]], device=DEV)
        return s
    rows, cols, top = case["rows"], case["cols"], case["top"]
    s["factor"] = -1.0 / TAU_SOFT if case["times"] else 1.0
    s["y"] = y = _outputs(case, gen)
    if case["op"] == "top":
        s.update(top_buffer=torch.empty(rows, top, device=DEV),
                 index_buffer=torch.empty(rows, top, dtype=torch.int32, device=DEV))
        return s
    # a teacher near the student; a few entries are unused, and one row in sixteen has no teacher
    z, none = _logits(s, y.float())
    z = z.add_(torch.randn(rows, cols, device=DEV, generator=gen))
    found = torch.topk(z.masked_fill_(none, -1e30), top, 1)
    index = found.indices.to(torch.int32)
    unused = (torch.rand(rows, top, device=DEV, generator=gen) < 0.05) | none.gather(1, found.indices)
    unused |= torch.rand(rows, 1, device=DEV, generator=gen) < 1.0 / 16
    s.update(top_in=found.values, index=index.masked_fill_(unused, -1),
             loss=torch.zeros(2, device=DEV), row_loss=torch.empty(rows, device=DEV),
             g=torch.empty(rows, cols, dtype=y.dtype, device=DEV))
    return s


# -- one pass --------------------------------------------------------------
def run(s):
    return (_run_own if own else _run_plain)(s)


def _run_own(s):
    from paper_2607_14672_gb300 import dstd
    if s["op"] == "quantize":
        dstd.quantize_mx4(s["x"], s["q"], s["scale"], s["values"])
        return s["values"]
    if s["op"] == "product":
        x = s["x_in"]
        if s["x"] != "codes":
            x = s["q"]
            dstd.quantize_mx4(s["x_in"], x, s["x_scale"])
        dstd.mx4_matmul(x, s["x_scale"], s["w"], s["w_scale"], s["out_buffer"])
        return s["out_buffer"]
    silent = T_END if s["times"] else None
    if s["op"] == "top":
        dstd.top_logits(s["y"], s["top_buffer"], s["index_buffer"], s["factor"], silent)
        return s["top_buffer"], s["index_buffer"]
    dstd.distill_loss(s["y"], s["top_in"], s["index"], s["loss"], s["row_loss"], s["g"], s["factor"], silent)
    return s["g"], s["row_loss"], s["loss"][:1]


def _run_plain(s):
    if s["op"] == "quantize":
        return _values(s["x"].float())
    if s["op"] == "product":
        cols = s["cols"]
        x = _unpacked(s["x_in"], s["x_scale"], cols) if s["x"] == "codes" else _values(s["x_in"].float())
        return (x @ _unpacked(s["w"], s["w_scale"], cols).t()).to(s["out_buffer"].dtype)
    z, none = _logits(s, s["y"].float())
    if s["op"] == "top":
        z, index = torch.sort(z, dim=1, descending=True, stable=True)
        return z[:, :s["top"]].contiguous(), index[:, :s["top"]].int()
    log_q = z - z.amax(1, keepdim=True)
    log_q = log_q - log_q.exp().sum(1, keepdim=True).log()
    used = s["index"] >= 0
    index = s["index"].clamp(min=0).long()
    v = s["top_in"].masked_fill(~used, -math.inf)
    v = v - v.amax(1, keepdim=True).clamp(min=-1e30)
    total = v.exp().sum(1, keepdim=True)
    p = v.exp() / total.clamp(min=1e-30)
    log_p = v - total.clamp(min=1e-30).log()
    rows = torch.where(used, p * (log_p - log_q.gather(1, index)), torch.zeros_like(p)).sum(1)
    g = log_q.exp().scatter_add(1, index, -p)
    g = (g * (s["factor"] / s["rows"])).masked_fill(none | (total == 0), 0.0)
    return g.to(s["g"].dtype), rows, rows.mean().reshape(1)


# -- from the definitions, in 64 bits ----------------------------------------
def _two_to(e):
    """2^e in 64 bits, from its bits."""
    return (e.long() + 1023 << 52).view(torch.float64)


def _exact_values(x):
    """Nearest code of each element, ties to the even code, by distance to every magnitude's midpoints."""
    rows, cols = x.shape
    out = torch.empty(rows, cols, dtype=torch.float64, device=x.device)
    level = torch.tensor(MAGNITUDES, dtype=torch.float64, device=x.device)
    middle = (level[1:] + level[:-1]) / 2
    step = max(1, (1 << 24) // cols)
    for i in range(0, rows, step):
        a = x[i:i + step].double()
        a = torch.cat((a, a.new_zeros(a.shape[0], -cols % BLOCK)), 1).unflatten(1, (-1, BLOCK))
        top = a.abs().max(2, keepdim=True).values
        e = torch.ceil(torch.log2(top.clamp(min=1e-60) / 6.0))
        e = torch.where(top > 6.0 * _two_to(e), e + 1, e)
        e = torch.where(top <= 6.0 * _two_to(e - 1), e - 1, e).clamp(min=-127)
        m = a.abs() * _two_to(-e)
        code = torch.bucketize(m, middle)          # a midpoint itself counts down
        tie = (code < 7) & (m == middle[code.clamp(max=6)]) & (code % 2 == 1)
        out[i:i + step] = (torch.sign(a) * level[code + tie.long()] * _two_to(e)).flatten(1)[:, :cols]
    return out


def _decoded(q, scale, cols):
    """Codes and exponents read one place after another."""
    rows, blocks = q.shape[0], q.shape[1] // 16
    level = torch.tensor(MAGNITUDES, dtype=torch.float64, device=q.device)
    r, b = torch.arange(rows, device=q.device)[:, None], torch.arange(blocks, device=q.device)
    place = ((r // 128) * ((blocks + 3) // 4) + b // 4) * 512 + (r % 32) * 16 + (r % 128 // 32) * 4 + b % 4
    power = _two_to(scale[place].int() - 127)
    out = torch.empty(rows, cols, dtype=torch.float64, device=q.device)
    step = max(1, (1 << 24) // cols)
    for i in range(0, rows, step):
        byte = q[i:i + step].long()
        code = torch.stack((byte % 16, byte // 16), 2).flatten(1)
        v = level[code % 8] * (1.0 - 2.0 * (code // 8))
        out[i:i + step] = (v.unflatten(1, (blocks, BLOCK)) * power[i:i + step, :, None]).flatten(1)[:, :cols]
    return out


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "quantize":
        return _exact_values(s["x"])
    if case["op"] == "product":
        cols = case["cols"]
        x = _decoded(s["x_in"], s["x_scale"], cols) if case["x"] == "codes" else _exact_values(s["x_in"])
        return torch.mm(x, _decoded(s["w"], s["w_scale"], cols).t())
    y, k = s["y"], case["top"]
    factor = float(torch.tensor(s["factor"], dtype=torch.float32))
    if case["op"] == "top":
        z = y.double() * factor
        if case["times"]:
            z[z == -math.inf] = factor * float(torch.tensor(T_END, dtype=torch.float32))
        return torch.topk(z, k, 1).values, None
    g = torch.zeros(case["rows"], case["cols"], dtype=torch.float64, device=DEV)
    rows = torch.zeros(case["rows"], dtype=torch.float64, device=DEV)
    step = max(1, (1 << 25) // case["cols"])
    for i in range(0, case["rows"], step):
        z = y[i:i + step].double() * factor
        none = torch.isneginf(z)
        if case["times"]:
            z[none] = factor * float(torch.tensor(T_END, dtype=torch.float32))
        log_q = torch.log_softmax(z, 1)
        at = s["index"][i:i + step].long()
        here = at >= 0
        taught = here.any(1, keepdim=True)
        v = torch.where(here, s["top_in"][i:i + step].double(), torch.full((), -math.inf, dtype=torch.float64, device=DEV))
        log_p = torch.where(taught, torch.log_softmax(v, 1), v)
        p = log_p.exp()
        rows[i:i + step] = torch.where(here, p * (log_p - log_q.gather(1, at.clamp(min=0))), p.new_zeros(())).sum(1)
        d = log_q.exp()
        d.scatter_add_(1, at.clamp(min=0), -torch.where(here, p, p.new_zeros(())))
        d[none | ~taught] = 0.0
        g[i:i + step] = d * (factor / case["rows"])
    return g, rows, rows.mean().reshape(1)


# -- what a pass cannot do without -------------------------------------------
def work(case):
    if case["op"] == "quantize":
        n = case["rows"] * case["cols"]
        return dict(bytes=int(n * (BYTES[case["type"]] + 17 / 32 + 4)), flops=4 * n)
    if case["op"] == "product":
        t, n, k = case["tokens"], case["rows"], case["cols"]
        read = n * k * 17 / 32 + t * k * (17 / 32 if case["x"] == "codes" else BYTES[case["x"]])
        return dict(bytes=int(read + t * n * BYTES[case["out"]]), flops=2 * t * n * k)
    n, k = case["rows"] * case["cols"], case["rows"] * case["top"]
    if case["op"] == "top":
        return dict(bytes=n * BYTES[case["type"]] + 8 * k, flops=2 * n)
    return dict(bytes=2 * n * BYTES[case["type"]] + 8 * k + 4 * case["rows"], flops=6 * n)

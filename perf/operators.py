"""Workloads of the operators of 8-bit training and serving: rows of weights and
of activations quantised to 8 bits, products of 8-bit rows with a scale for each
token and channel, and the optimiser's side of a training step (many gradients
clipped by their global norm, and the clipped AdamW update).

A case is a dict of plain values; ``listed`` gives the named ones, ``draw``
more of the same ranges. ``run`` is one pass: with ``own`` through the
framework's entry points, otherwise in elementary torch operations.
"""

import math

import torch

own = False

DEV = "cuda"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
BYTES = {"f32": 4, "bf16": 2, "int8": 1}
LR, B1, B2, EPS, DECAY, MAX_NORM = 1e-3, 0.9, 0.999, 1e-8, 1e-2, 1.0

# parameter tensors of the repository's networks: the MLP 784-800-800-10 and the 20-layer conv network
MLP = "627200 640000 8000"
CONV20 = " ".join(["576"] + ["36864"] * 5 + ["73728"] + ["147456"] * 6 + ["294912"] + ["589824"] * 5 + ["125440"])


def listed():
    return [
        # the MLP's first layer before a training step's forward: codes, scales and the values the codes stand for
        dict(name="quantize mlp weights", op="quantize", rows=800, cols=784, type="f32", pad=0),
        # the largest dense layer's weights
        dict(name="quantize 16k weights", op="quantize", rows=16384, cols=16384, type="f32", pad=0),
        # the smallest call: one token through one layer, where latency counts
        dict(name="product 1 token", op="product", tokens=1, cols=4096, rows=4096, x="int8", out="f32", pad=0),
        # one sample of 8 grid points through the largest dense layer, where reading the weights counts
        dict(name="product 8 tokens 16k", op="product", tokens=8, cols=16384, rows=16384, x="int8", out="bf16", pad=0),
        # odd sizes and padded rows: one sample of 37 grid points, activations quantised on the way
        dict(name="product odd", op="product", tokens=37, cols=1023, rows=801, x="f32", out="f32", pad=9),
        # the MLP's first layer on its training batch: 256 samples of 32 grid points
        dict(name="product mlp batch", op="product", tokens=8192, cols=784, rows=800, x="f32", out="f32", pad=0),
        # the largest dense layer: 128 samples of 32 grid points
        dict(name="product 16k batch", op="product", tokens=4096, cols=16384, rows=16384, x="bf16", out="f32", pad=0),
        # the MLP's gradients at odd places of one buffer
        dict(name="clip mlp odd", op="clip", sizes=MLP, type="f32", gap=1),
        # 16-bit gradients of the largest dense layer and its readout
        dict(name="clip 16k", op="clip", sizes="268435456 163840", type="bf16", gap=0),
        # an optimiser step of the MLP
        dict(name="step mlp", op="step", sizes=MLP, type="f32", gap=0),
        # of the 20-layer conv network
        dict(name="step conv20", op="step", sizes=CONV20, type="f32", gap=0),
        # of the largest dense layer and its readout, with 16-bit gradients
        dict(name="step 16k", op="step", sizes="268435456 163840", type="bf16", gap=0),
    ]


def _spread(rng, low, high):
    """A whole number of [low, high], spread over its logarithm."""
    return min(high, max(low, int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))))


def draw(rng):
    op = rng.choice(["quantize", "product", "product", "product", "clip", "step"])
    if op == "quantize":
        return dict(op=op, rows=_spread(rng, 1, 16384), cols=_spread(rng, 8, 16384), type=rng.choice(["f32", "bf16"]),
                    pad=rng.choice([0, 0, rng.randint(1, 17)]))
    if op == "product":
        cols, rows = _spread(rng, 16, 16384), _spread(rng, 8, 16384)
        tokens = _spread(rng, 1, 16384)
        tokens = max(1, min(tokens, 4096 * 16384 * 16384 // (cols * rows), (1 << 27) // rows, (1 << 27) // cols))
        return dict(op=op, tokens=tokens, cols=cols, rows=rows, x=rng.choice(["int8", "f32", "bf16"]),
                    out=rng.choice(["f32", "bf16"]), pad=rng.choice([0, 0, rng.randint(1, 17)]))
    sizes, left = [], 1 << 28
    for _ in range(rng.randint(1, 24)):
        n = min(left, _spread(rng, 1, 1 << 26))
        if n:
            sizes.append(n)
            left -= n
    return dict(op=op, sizes=" ".join(map(str, sizes)), type=rng.choice(["f32", "bf16"]), gap=rng.choice([0, 0, 1, 3]))


# -- inputs ----------------------------------------------------------------
def _generator(seed):
    return torch.Generator(device=DEV).manual_seed(int(seed))


def _padded(rows, cols, pad, dtype):
    return torch.empty(rows, cols + pad, dtype=dtype, device=DEV)[:, :cols]


def _weights(case, gen):
    """W = mu + N(0, 1/fan_in) with mu fan_in = 12, as the dense layers are initialised."""
    rows, cols = case["rows"], case["cols"]
    return torch.randn(rows, cols, device=DEV, generator=gen).mul_(1.0 / math.sqrt(cols)).add_(12.0 / cols)


def _grid_weights(case, gen):
    """Activations of a layer: most inputs carry no weight at a given grid point."""
    x = torch.rand(case["tokens"], case["cols"], device=DEV, generator=gen)
    kept = torch.rand(case["tokens"], case["cols"], device=DEV, generator=gen) < 0.2
    return x.mul_(kept)


def _codes(x):
    """8-bit codes of each row and their scales, to make inputs with."""
    top = x.abs().amax(1, keepdim=True).clamp_(min=1e-20)
    return torch.round(x * (127.0 / top)).to(torch.int8), (top / 127.0).reshape(-1)


def _places(case):
    """(size, start in the flat buffer) of each tensor, and the buffer's length."""
    at, found = case["gap"], []
    for n in map(int, case["sizes"].split()):
        found.append((n, at))
        at += n + case["gap"]
    return found, at


def _flat(case, dtype, fill):
    """A flat buffer with the tensors at their places and zeros between them."""
    places, total = _places(case)
    flat = torch.zeros(total, dtype=dtype, device=DEV)
    for n, at in places:
        flat[at:at + n] = fill(n)
    return flat, [flat[at:at + n] for n, at in places]


def prepare(case, seed):
    gen = _generator(seed)
    s = dict(case)
    if case["op"] == "quantize":
        x = _padded(case["rows"], case["cols"], case["pad"], TYPES[case["type"]])
        x.copy_(_weights(case, gen))
        s.update(x=x, q=torch.empty(case["rows"], case["cols"], dtype=torch.int8, device=DEV),
                 scale=torch.empty(case["rows"], device=DEV), values=torch.empty(case["rows"], case["cols"], device=DEV))
        return s
    if case["op"] == "product":
        tokens, rows, cols, pad = case["tokens"], case["rows"], case["cols"], case["pad"]
        w = _padded(rows, cols, pad, torch.int8)
        codes, w_scale = _codes(_weights(case, gen))
        w.copy_(codes)
        x = _grid_weights(case, gen)
        s.update(w=w, w_scale=w_scale, out_buffer=torch.empty(tokens, rows, dtype=TYPES[case["out"]], device=DEV))
        if case["x"] == "int8":
            codes, s["x_scale"] = _codes(x)
            s["x_in"] = _padded(tokens, cols, pad, torch.int8)
            s["x_in"].copy_(codes)
        else:
            s["x_in"] = _padded(tokens, cols, pad, TYPES[case["x"]])
            s["x_in"].copy_(x)
            s["q"] = torch.empty(tokens, cols, dtype=torch.int8, device=DEV)
            s["x_scale"] = torch.empty(tokens, device=DEV)
        if own:  # scratch of the size that the framework asks for
            from paper_2607_14672_gb300 import dstd
            s["workspace"] = torch.empty(dstd.int8_matmul_workspace_bytes(tokens, rows, cols), dtype=torch.uint8, device=DEV)
        return s
    size = 10.0 ** (torch.rand(1, generator=gen, device=DEV).item() - 2.0)
    s["g"], gs = _flat(case, TYPES[case["type"]], lambda n: torch.randn(n, device=DEV, generator=gen) * size)
    s["norm"] = torch.zeros(1, device=DEV)
    lists = [gs]
    if case["op"] == "clip":
        s["out_flat"], outs = _flat(case, TYPES[case["type"]], lambda n: torch.zeros(n, device=DEV))
        lists.append(outs)
    else:
        s["w"], ws = _flat(case, torch.float32, lambda n: torch.randn(n, device=DEV, generator=gen) * 0.03)
        s["m"], ms = _flat(case, torch.float32, lambda n: torch.randn(n, device=DEV, generator=gen) * 1e-3)
        s["v"], vs = _flat(case, torch.float32, lambda n: torch.rand(n, device=DEV, generator=gen) * 1e-6)
        s["count"] = torch.tensor([10, 0], dtype=torch.int32, device=DEV)
        lists = [ws, gs, ms, vs]
    if own:  # what a training program keeps: its tensor lists and the norm's scratch
        from paper_2607_14672_gb300 import dstd
        s["lists"] = [dstd.TensorList(t) for t in lists]
        s["workspace"] = torch.zeros(dstd.grad_norm_workspace_bytes(gs), dtype=torch.uint8, device=DEV)
    return s


# -- one pass --------------------------------------------------------------
def run(s):
    return (_run_own if own else _run_plain)(s)


def _run_own(s):
    from paper_2607_14672_gb300 import dstd
    if s["op"] == "quantize":
        dstd.quantize_rows(s["x"], s["q"], s["scale"], s["values"])
        return s["values"], s["scale"]
    if s["op"] == "product":
        x = s["x_in"]
        if s["x"] != "int8":
            x = s["q"]
            dstd.quantize_rows(s["x_in"], x, s["x_scale"])
        dstd.int8_matmul(x, s["x_scale"], s["w"], s["w_scale"], s["out_buffer"], s["workspace"])
        return s["out_buffer"]
    if s["op"] == "clip":
        gs, outs = s["lists"]
        dstd.clip_grads(gs, MAX_NORM, s["norm"], s["workspace"], outs)
        return s["out_flat"], s["norm"]
    ws, gs, ms, vs = s["lists"]
    dstd.adamw_clip(ws, gs, ms, vs, LR, B1, B2, EPS, DECAY, s["count"], MAX_NORM, s["norm"], s["workspace"])
    return s["w"], s["m"], s["v"], s["count"][:1], s["norm"]


def _plain_codes(x):
    top = x.abs().amax(1, keepdim=True)
    inverse = torch.where(top > 0, 127.0 / top, torch.zeros_like(top))
    return torch.round(x * inverse), top / 127.0


def _plain_clip(g):
    norm = g.square().sum().sqrt().reshape(1)
    return g * torch.where(norm > MAX_NORM, MAX_NORM / norm, torch.ones_like(norm)), norm


def _run_plain(s):
    if s["op"] == "quantize":
        q, scale = _plain_codes(s["x"].float())
        return q * scale, scale.reshape(-1)
    if s["op"] == "product":
        x = s["x_in"].float()
        scale = s["x_scale"].reshape(-1, 1)
        if s["x"] != "int8":
            x, scale = _plain_codes(x)
        return ((x @ s["w"].float().t()) * scale * s["w_scale"]).to(s["out_buffer"].dtype)
    g, norm = _plain_clip(s["g"].float())
    if s["op"] == "clip":
        return g.to(s["g"].dtype), norm
    s["count"][0] += 1
    t = s["count"][:1].float()
    unbias1, unbias2 = -torch.expm1(t * math.log(B1)), -torch.expm1(t * math.log(B2))
    w, m, v = s["w"], s["m"], s["v"]
    m.mul_(B1).add_(g * (1.0 - B1))
    v.mul_(B2).add_(g.square() * (1.0 - B2))
    w.mul_(1.0 - LR * DECAY).sub_(LR * (m / unbias1) / ((v / unbias2).sqrt() + EPS))
    return w, m, v, s["count"][:1], norm


# -- from the definitions, in 64 bits ----------------------------------------
def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "quantize":
        x = s["x"].double()
        step = x.abs().max(dim=1).values / 127.0
        each = step.clamp(min=1e-300)[:, None]
        return torch.round(x / each) * each, step
    if case["op"] == "product":
        if case["x"] == "int8":
            x, step = s["x_in"].double(), s["x_scale"].double()
        else:
            x = s["x_in"].double()
            step = x.abs().max(dim=1).values / 127.0
            x = torch.round(x / step.clamp(min=1e-300)[:, None])
        sums = torch.mm(x, s["w"].double().t())
        return sums.mul_(step[:, None]).mul_(s["w_scale"].double()[None, :])
    g = s["g"].double()
    norm = torch.linalg.vector_norm(g).reshape(1)
    g = g * min(1.0, MAX_NORM / norm.item())
    if case["op"] == "clip":
        return g, norm
    t = int(s["count"][0].item()) + 1
    m = B1 * s["m"].double() + (1 - B1) * g
    v = B2 * s["v"].double() + (1 - B2) * g * g
    change = (m / (1 - B1 ** t)) / (torch.sqrt(v / (1 - B2 ** t)) + EPS)
    w = s["w"].double() * (1 - LR * DECAY) - LR * change
    return w, m, v, None, norm


# -- what a pass cannot do without -------------------------------------------
def work(case):
    if case["op"] == "quantize":
        n = case["rows"] * case["cols"]
        return dict(bytes=n * (BYTES[case["type"]] + 1 + 4) + 4 * case["rows"], flops=4 * n)
    if case["op"] == "product":
        t, n, k = case["tokens"], case["rows"], case["cols"]
        read = t * k * BYTES[case["x"]] + n * k + 4 * n + (4 * t if case["x"] == "int8" else 0)
        return dict(bytes=read + t * n * BYTES[case["out"]], flops=2 * t * n * k)
    n, e = sum(map(int, case["sizes"].split())), BYTES[case["type"]]
    if case["op"] == "clip":
        return dict(bytes=2 * n * e + 4, flops=3 * n)
    return dict(bytes=n * (e + 24) + 16, flops=16 * n)

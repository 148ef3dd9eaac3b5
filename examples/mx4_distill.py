"""Train the 784-800-800-10 network for 4-bit weights from a teacher, and serve it in 4 bits.

    python examples/mx4_distill.py [--steps 24] [--batch 64] [--top 4] [--weight 1.0]

A network of the same layers is trained first, in the three-product mode, and keeps its largest output
logits of each sample: the record. The 4-bit network starts from other weights and learns from the labels
and from that record: every step quantises the weights in blocks of 32, runs the layers' products on the
4-bit tensor cores, adds the distillation loss's gradient to the cross-entropy's, passes it straight through
the rounding, and updates the fp32 weights with AdamW; the step is captured once in a CUDA graph. Then a
network of batch 1 takes over the codes alone and answers single samples. Data are synthetic (seeded
intensities, random labels).
"""

import argparse
import os
import sys

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)

import torch  # noqa: E402

from paper_2607_14672_gb300 import configs, dstd, net  # noqa: E402


def captured_steps(n, steps):
    """Cross-entropies, and distillation losses where there is a teacher, of captured training steps."""
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        n.step(stream)                       # outside the capture: the library's first launches
    seen = [(n.loss[0].item(), float(n.taught_value()))]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        n.step(stream)
    for _ in range(steps - 1):
        graph.replay()
        seen.append((n.loss[0].item(), float(n.taught_value())))
    torch.cuda.synchronize()
    return seen


def teacher_record(cfg, steps, top):
    """The largest logits of a trained network and their classes."""
    n = net.DenseNet(cfg, "x3", with_adamw=True, max_norm=0.5)
    n.set_inputs(cfg["inputs"](B=n.B), cfg["labels"](B=n.B))
    captured_steps(n, steps)
    n.forward()
    logits = torch.empty(n.B, top, device="cuda")
    classes = torch.empty(n.B, top, dtype=torch.int32, device="cuda")
    n.answers(logits, classes)
    return logits, classes


def train(cfg, steps, record, weight):
    n = net.DenseNet(cfg, "mx4", with_adamw=True, max_norm=0.5)
    gen = torch.Generator(device="cuda").manual_seed(1)
    for w in n.W:
        w.add_(torch.randn(w.shape, generator=gen, device="cuda") * 0.3 * w.std())
    n.set_inputs(cfg["inputs"](B=n.B), cfg["labels"](B=n.B))
    n.learn_from(record[0].shape[1], weight=weight)
    n.set_teacher(*record)
    losses = captured_steps(n, steps)
    n.quantize()                             # the codes of the last update's weights
    return n, losses


def serve(cfg, trained, samples):
    """Spike times of single samples from the codes alone."""
    one = net.DenseNet(configs.config2(batch=1), "mx4")
    one.take_codes(trained)
    times = []
    for x in cfg["inputs"](B=trained.B)[:samples]:
        one.set_inputs(x[None])
        one.serve()
        times.append(one.t[-1].clone())
    return torch.cat(times)


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--steps", type=int, default=24)
    ap.add_argument("--batch", type=int, default=64)
    ap.add_argument("--top", type=int, default=4)
    ap.add_argument("--weight", type=float, default=1.0)
    a = ap.parse_args(argv)
    cfg = configs.config2(batch=a.batch)
    record = teacher_record(cfg, a.steps, a.top)
    n, losses = train(cfg, a.steps, record, a.weight)
    for i in range(0, a.steps, max(1, a.steps // 8)):
        print(f"step {i:3d}  cross entropy {losses[i][0]:.4f}  distillation loss {losses[i][1]:.4f}")
    n.serve()
    alone = serve(cfg, n, 8)
    torch.cuda.synchronize()
    if dstd.device_status() != 0:
        raise RuntimeError("a device-side wait expired")
    batched = n.t[-1][:8]
    both = torch.isfinite(alone) & torch.isfinite(batched)
    off = (alone - batched)[both].abs().max().item() if both.any() else 0.0
    print(f"8 samples served one by one: spike times within {off:.1e} of those in the batch; "
          f"earliest outputs {alone.argmin(1).tolist()}")
    return losses, off


if __name__ == "__main__":
    main()

"""Train the 784-800-800-10 network for 8-bit weights and serve it in 8 bits.

    python examples/q8_mlp.py [--steps 24] [--batch 64] [--max-norm 0.5]

Every training step quantises the weights by rows, runs the layers' products on
8-bit codes, passes the gradient straight through the rounding, and updates the
fp32 weights with AdamW on gradients clipped to a global norm; the step is
captured once in a CUDA graph. Then a second network of batch 1 takes over the
codes alone and answers single samples, and its answers are compared with the
training network's. Data are synthetic (seeded intensities, random labels).
"""

import argparse
import os
import sys

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)

import torch  # noqa: E402

from paper_2607_14672_gb300 import configs, dstd, net  # noqa: E402


def train(steps, batch, max_norm):
    cfg = configs.config2(batch=batch)
    n = net.DenseNet(cfg, "q8", with_adamw=True, max_norm=max_norm)
    n.set_inputs(cfg["inputs"](B=batch), cfg["labels"](B=batch))
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        n.step(stream)                       # outside the capture: the library's first launches
    losses, norms = [n.loss[0].item()], [n.grad_norm.item()]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        n.step(stream)
    for _ in range(steps - 1):
        graph.replay()
        losses.append(n.loss[0].item())
        norms.append(n.grad_norm.item())
    torch.cuda.synchronize()
    n.quantize()                             # the codes of the last update's weights
    return cfg, n, losses, norms


def serve(cfg, trained, samples):
    """Spike times of single samples from the codes alone."""
    one = net.DenseNet(configs.config2(batch=1), "q8")
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
    ap.add_argument("--max-norm", type=float, default=0.5)
    a = ap.parse_args(argv)
    cfg, n, losses, norms = train(a.steps, a.batch, a.max_norm)
    for i in range(0, a.steps, max(1, a.steps // 8)):
        print(f"step {i:3d}  cross entropy {losses[i]:.4f}  gradient norm {norms[i]:.3f}")
    n.serve()
    alone = serve(cfg, n, 8)
    torch.cuda.synchronize()
    if dstd.device_status() != 0:
        raise RuntimeError("a device-side wait expired")
    batched = n.t[-1][:8]
    same = torch.equal(alone, batched)
    print(f"8 samples served one by one: {'the same spike times as' if same else 'NOT the same as'} in the batch; "
          f"earliest outputs {alone.argmin(1).tolist()}")
    return losses, same


if __name__ == "__main__":
    main()

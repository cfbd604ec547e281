"""Data-parallel training of a small network with the whole set of operators:

* every worker runs its layers' products, forward and backward, in 8-bit integers (``Int8Linear``) and writes the gradients
  of its weights straight into its row of the flat gradient [n, d];
* the rows go through DoubleSqueeze (1-bit compression with error compensation on both passes), which gives Q[v];
* each weight matrix moves by the orthogonalised momentum of its slice of Q[v] (``OrthUpdate``).

The task is a fixed random teacher network.  Run:  python examples/train_int8_orth.py [steps]
"""
from __future__ import annotations

import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_1905_05957_b200 import DoubleSqueeze, Int8Linear, OrthUpdate, Q, device_status  # noqa: E402


def train(steps: int = 60, workers: int = 4, batch: int = 256, width: int = 192, rate: float = 0.03, seed: int = 0) -> list[float]:
    """Mean loss over the workers at every step."""
    gen = torch.Generator(device="cuda").manual_seed(seed)

    def normal(*shape):
        return torch.randn(*shape, device="cuda", generator=gen)

    inputs, outputs = 64, 32
    shapes = [(width, inputs), (width, width), (outputs, width)]
    sizes = [o * i for o, i in shapes]
    starts = [sum(sizes[:k]) for k in range(len(sizes))]
    d = sum(sizes)
    teacher = [normal(o, i) / i ** 0.5 for o, i in shapes]
    model = torch.cat([(normal(o, i) / i ** 0.5).reshape(-1) for o, i in shapes])
    momentum = torch.zeros(d, device="cuda")

    def slices(v):
        return [v[s:s + n].view(shape) for s, n, shape in zip(starts, sizes, shapes)]

    # gamma = -1 on a model of zeros: x becomes Q[v] itself, the compressed mean gradient
    step = DoubleSqueeze(workers, d, -1.0, Q("sign1", chunk=4096), Q("sign1", chunk=4096), seed)
    plans = [OrthUpdate(o, i, momentum=0.9) for o, i in shapes]
    g = torch.empty(workers, d, device="cuda")
    losses = []
    for t in range(steps):
        layers = [Int8Linear(w) for w in slices(model)]
        total = torch.zeros((), device="cuda")
        for w in range(workers):
            x = normal(batch, inputs).to(torch.bfloat16)
            target = x.float()
            for k, m in enumerate(teacher):
                target = target @ m.T
                if k + 1 < len(teacher):
                    target = torch.relu(target)
            hidden = [x]
            for k, layer in enumerate(layers):
                y = layer.forward(hidden[-1], training=True)
                hidden.append(torch.relu(y) if k + 1 < len(layers) else y)
            diff = hidden[-1].float() - target
            total += diff.square().mean()
            dy = (2 / diff.numel() * diff).to(torch.bfloat16)
            grads = slices(g[w])
            for k in reversed(range(len(layers))):
                dx, _, _ = layers[k].backward(dy, dw=grads[k])
                dy = dx * (hidden[k] > 0) if k else None
        step.x.zero_()
        step.step(g, t)
        for plan, q, m, w in zip(plans, slices(step.x), slices(momentum), slices(model)):
            plan.update(q, m, out_dtype=None, x=w, gamma=rate * (1 - t / steps))
        losses.append(total / workers)
    losses = [float(v) for v in losses]
    step.close()
    if device_status() or any(plan.timed_out() for plan in plans):      # a product that gave up waiting leaves wrong numbers
        raise RuntimeError("a matrix product timed out on the device")
    return losses


if __name__ == "__main__":
    got = train(int(sys.argv[1]) if len(sys.argv) > 1 else 200)
    for t in range(0, len(got), max(1, len(got) // 10)):
        print(f"step {t:4d}  loss {got[t]:.4f}")
    print(f"last       loss {got[-1]:.4f}")

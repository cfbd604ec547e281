"""Data-parallel training of a residual network in 16-bit floats, its gradients compressed by the step:

* every worker runs blocks of  n = pre(h), y = W2 gelu(W1 n + b1) + b2, h = h + D(g y)  with the layers' products in bf16 (``Linear16``), the residual
  stream in 32 bits and what stands between the blocks in one operator (``ResidualNorm``, dropout included), and writes every gradient straight into its
  row of the flat gradient [n, d];
* the rows go through DoubleSqueeze (1-bit compression with error compensation on both passes), which moves the model.

The task is a fixed random teacher.  Run:  python examples/train_residual16.py [steps]
"""
from __future__ import annotations

import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_1905_05957_b200 import DoubleSqueeze, Linear16, Q, ResidualNorm, device_status, dropout  # noqa: E402

SCALE = 1.0


def shapes(width: int, hidden: int, blocks: int) -> dict[str, tuple[int, ...]]:
    """Parameters by name, in the order in which they lie in the flat model."""
    s = {}
    for k in range(blocks):
        s |= {f"{k}.norm": (width,), f"{k}.w1": (hidden, width), f"{k}.b1": (hidden,), f"{k}.w2": (width, hidden), f"{k}.b2": (width,), f"{k}.gate": (width,)}
    return s | {"norm": (width,)}


def views(flat: torch.Tensor, names: dict[str, tuple[int, ...]]) -> dict[str, torch.Tensor]:
    out, at = {}, 0
    for name, shape in names.items():
        n = 1
        for v in shape:
            n *= v
        out[name] = flat[at:at + n].view(shape)
        at += n
    return out


class Network:
    """The blocks, made of views of a flat model in 32 bits."""

    def __init__(self, model: dict[str, torch.Tensor], blocks: int, p: float, seed: int):
        self.p, self.seed, self.first = p, seed, ResidualNorm("layer", pre_weight=model["0.norm"])
        self.layers, self.joints = [], []
        for k in range(blocks):
            self.layers.append((Linear16(model[f"{k}.w1"], model[f"{k}.b1"], "gelu"), Linear16(model[f"{k}.w2"], model[f"{k}.b2"])))
            after = model[f"{k + 1}.norm"] if k + 1 < blocks else model["norm"]
            self.joints.append(ResidualNorm("layer", gate=model[f"{k}.gate"], pre_weight=after, residual_scale=SCALE, p=p, seed=seed, layer=k))

    def forward(self, x: torch.Tensor, step: int) -> torch.Tensor:
        """x [tokens, width] in 32 bits -> the last norm's output in bf16."""
        x16 = dropout(x, self.p, self.seed, step=step, layer=1000).to(torch.bfloat16)
        h, n = self.first.forward(x16, training=True, h=torch.empty_like(x))
        for (w1, w2), joint in zip(self.layers, self.joints):
            y = w2.forward(w1.forward(n, training=True), training=True)
            h, n = joint.forward(y, h, step=step, training=True)
        return n

    def backward(self, dn: torch.Tensor, grads: dict[str, torch.Tensor]):
        """Every parameter's gradient into its view."""
        dh, last = None, "norm"
        for k in reversed(range(len(self.layers))):
            dy, dh, _ = self.joints[k].backward(dh, dn, out={"gate": grads[f"{k}.gate"], "pre_weight": grads[last]})
            w1, w2 = self.layers[k]
            da, _, _ = w2.backward(dy, dw=grads[f"{k}.w2"], db=grads[f"{k}.b2"])
            dn, _, _ = w1.backward(da, dw=grads[f"{k}.w1"], db=grads[f"{k}.b1"])
            last = f"{k}.norm"
        self.first.backward(dh, dn, out={"pre_weight": grads[last]})


def start(names: dict[str, tuple[int, ...]], seed: int) -> torch.Tensor:
    gen = torch.Generator(device="cuda").manual_seed(seed)
    parts = []
    for name, shape in names.items():
        if len(shape) == 2:
            parts.append((torch.randn(shape, device="cuda", generator=gen) / shape[1] ** 0.5).reshape(-1))
        else:
            parts.append(torch.full(shape, 0.0 if ".b" in name else 0.5 if "gate" in name else 1.0, device="cuda"))
    return torch.cat(parts)


def train(steps: int = 40, workers: int = 4, tokens: int = 256, width: int = 96, hidden: int = 200, blocks: int = 2, rate: float = 0.05, p: float = 0.1,
          seed: int = 0) -> list[float]:
    """Mean loss over the workers at every step."""
    names = shapes(width, hidden, blocks)
    model = start(names, seed)
    gen = torch.Generator(device="cuda").manual_seed(seed + 1)
    teacher = torch.randn(width, width, device="cuda", generator=gen) / width ** 0.5
    ds = DoubleSqueeze(workers, model.numel(), rate, Q("sign1", chunk=1024), Q("sign1", chunk=1024), seed)
    ds.x.copy_(model)
    g = torch.empty(workers, model.numel(), device="cuda")
    losses = []
    for t in range(steps):
        total = torch.zeros((), device="cuda")
        for w in range(workers):
            net = Network(views(ds.x, names), blocks, p, seed + w)
            x = torch.randn(tokens, width, device="cuda", generator=gen)
            n = net.forward(x, t)
            diff = n.float() - torch.tanh(x @ teacher.T)
            total += diff.square().mean()
            net.backward((2 / diff.numel() * diff).to(torch.bfloat16), views(g[w], names))
        ds.step(g, t)
        losses.append(total / workers)
    losses = [float(v) for v in losses]
    ds.close()
    if device_status():      # a product that gave up waiting leaves wrong numbers
        raise RuntimeError("a matrix product timed out on the device")
    return losses


if __name__ == "__main__":
    got = train(int(sys.argv[1]) if len(sys.argv) > 1 else 200)
    for t in range(0, len(got), max(1, len(got) // 10)):
        print(f"step {t:4d}  loss {got[t]:.4f}")
    print(f"last       loss {got[-1]:.4f}")

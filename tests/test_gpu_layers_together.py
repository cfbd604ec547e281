"""The 16-bit layers, the norms and dropout as they are used together: a network's gradients against those of the same network in 64 bits, the example, streams,
graphs, and sizes that reach every form of the product."""
import importlib.util
import os

import pytest
import torch

from paper_1905_05957_b200 import Linear16, ResidualNorm, dropout, layer_ops, linear16, matrix_ops
from tests.test_gpu_dropout import kept

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def _example():
    spec = importlib.util.spec_from_file_location("train_residual16", os.path.join(ROOT, "examples", "train_residual16.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def _normal(*shape, seed, dtype=torch.float32, scale=1.0):
    return (scale * torch.randn(*shape, device="cuda", generator=torch.Generator(device="cuda").manual_seed(seed))).to(dtype)


def test_gradients_of_the_example():
    """Every parameter's gradient, in a row of the step, against autograd in 64 bits.  Weights, activations, z and dz are rounded to bf16 (half a step 2^-9 each), some thirty
    times along the two blocks and back; errors of random sign add up as their squares: 2^-9 sqrt(30) = 1.1 %, of which a tensor's norm may be off by 3 % here."""
    ex = _example()
    width, hidden, blocks, tokens, p, seed, step = 40, 72, 2, 64, 0.2, 9, 3
    names = ex.shapes(width, hidden, blocks)
    flat = ex.start(names, 1) + 0.05 * _normal(sum(torch.Size(s).numel() for s in names.values()), seed=2)
    x, dn = _normal(tokens, width, seed=3), _normal(tokens, width, seed=4, dtype=torch.bfloat16)
    g = torch.full((2, flat.numel()), 7.0, device="cuda")
    net = ex.Network(ex.views(flat, names), blocks, p, seed)
    n = net.forward(x, step)
    net.backward(dn, ex.views(g[1], names))
    assert bool((g[0] == 7.0).all())

    m = {k: v.double().requires_grad_() for k, v in ex.views(flat, names).items()}
    keep = 65536 / (65536 - round(p * 65536))

    def norm(v, w):
        return torch.nn.functional.layer_norm(v, (width,), eps=1e-5) * w
    h = torch.where(kept(tokens, width, p, seed, step, 1000), x.double() * keep, 0.0)
    a = norm(h, m["0.norm"])
    for k in range(blocks):
        y = torch.nn.functional.gelu(a @ m[f"{k}.w1"].T + m[f"{k}.b1"]) @ m[f"{k}.w2"].T + m[f"{k}.b2"]
        h = ex.SCALE * h + torch.where(kept(tokens, width, p, seed, step, k), y * m[f"{k}.gate"] * keep, 0.0)
        a = norm(h, m[f"{k + 1}.norm"] if k + 1 < blocks else m["norm"])
    assert float((n.double() - a.detach()).norm() / a.detach().norm()) < 0.03
    want = torch.autograd.grad(a, list(m.values()), dn.double())
    for (name, got), ref in zip(ex.views(g[1], names).items(), want):
        assert float((got.double() - ref).norm() / ref.norm()) < 0.03, name


def test_the_example_runs_and_repeats():
    ex = _example()
    losses = ex.train(steps=6)
    assert len(losses) == 6 and all(v == v and v < 100 for v in losses)
    assert ex.train(steps=3) == losses[:3]                # nothing depends on the order of threads


# reached by size on a B200: tiles of 64, 128, 192 and 256 columns, pairs of CTAs, K split by 2, 4 and 8, the same with the operands' places exchanged
FORMS = [(130, 640, 520), (640, 384, 640), (1500, 256, 1480), (2304, 512, 2304), (4096, 512, 4096), (4000, 128, 6000), (256, 8192, 128), (256, 4096, 512), (512, 4096, 1024),
         (512, 9000, 513), (1000, 2000, 3001), (64, 16384, 64), (48, 4096, 1000), (24, 8192, 4096), (30, 300, 20000), (12, 8000, 9000)]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("m,k,n", FORMS)
def test_every_form_is_exact(m, k, n, dtype):
    """Whole numbers, whose sums are exact in 32 bits: forward with bias and residual, gradients in 16 and 32 bits."""
    gen = torch.Generator(device="cuda").manual_seed(m + n)
    x, w, r, dy = (torch.randint(-2, 3, s, device="cuda", generator=gen).to(dtype) for s in ((m, k), (n, k), (m, n), (m, n)))
    b = torch.randint(-9, 10, (n,), device="cuda", generator=gen).float()
    z = x.double() @ w.double().T + b
    assert torch.equal(linear16(x, w, b, residual=r), (z + r.double()).to(dtype))
    assert torch.equal(linear16(x, w, b, "relu", out_dtype=torch.float32), torch.relu(z).float())
    layer = Linear16(w, b, "relu")
    assert torch.equal(layer.forward(x, residual=r, training=True), (torch.relu(z) + r.double()).to(dtype))
    dz = dy.double() * (z > 0)
    dx, dw, db = layer.backward(dy, grad_dtype=torch.float32)
    assert torch.equal(dx, (dz @ w.double()).to(dtype)) and torch.equal(dw, (dz.T @ x.double()).float()) and torch.equal(db, dz.sum(0).float())
    _, dw, _ = layer.backward(dy, need_dx=False)
    assert torch.equal(dw, (dz.T @ x.double()).to(dtype))


def _block(width, hidden, dtype=torch.bfloat16):
    w1, w2 = _normal(hidden, width, seed=1, dtype=dtype, scale=width ** -0.5), _normal(width, hidden, seed=2, dtype=dtype, scale=hidden ** -0.5)
    b1, norm, gate = _normal(hidden, seed=3), 1 + _normal(width, seed=4, scale=0.1), _normal(width, seed=5)

    def step(x, dh, p=0.1):
        """What a training step of one block calls, its results."""
        before = ResidualNorm("rms", pre_weight=norm)
        l1, l2 = Linear16(w1, b1, "silu"), Linear16(w2)
        after = ResidualNorm("layer", post_weight=norm, gate=gate, pre_weight=norm, p=p, seed=5)
        _, n = before.forward(x, training=True, need_h=False)
        y = l2.forward(dropout(l1.forward(n, training=True), p, 6), training=True)
        h, out = after.forward(y, x, training=True)
        dy, dx, g1 = after.backward(dh, dh)
        da, dw2, _ = l2.backward(dy)
        dn, dw1, db1 = l1.backward(dropout(da, p, 6))
        dx2, _, g2 = before.backward(dn=dn)
        return [h, out, dx, dx2, dw1, dw2, db1, *g1.values(), *g2.values()]
    return step


@pytest.mark.parametrize("rows,width,hidden", [(1, 64, 96), (40, 100, 77), (300, 520, 1032)])
def test_a_step_captured_before_any_other(rows, width, hidden, monkeypatch):
    step = _block(width, hidden)
    x, dh = _normal(rows, width, seed=7, dtype=torch.bfloat16), _normal(rows, width, seed=8, dtype=torch.bfloat16)
    want = [t.clone() for t in step(x, dh)]
    torch.cuda.synchronize()
    monkeypatch.setattr(matrix_ops, "_status", {})      # as a process starts
    monkeypatch.setattr(layer_ops, "_status", matrix_ops._status)
    graphs, got = [], []
    for _ in range(2):                                  # two graphs of one step: neither has anything of the other's
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            got.append(step(x, dh))
    for i in (0, 1, 0):
        for t in got[i]:
            t.fill_(float("nan"))
        graphs[i].replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got[i], want))
    x.mul_(2)                                           # replays read what is there then
    again = [t.clone() for t in step(x, dh)]
    graphs[1].replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got[1], again))


def test_a_graph_replayed_while_others_run():
    step = _block(256, 520)
    x, dh = _normal(500, 256, seed=7, dtype=torch.bfloat16), _normal(500, 256, seed=8, dtype=torch.bfloat16)
    want = [t.clone() for t in step(x, dh)]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step(x, dh)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for _ in range(10):
        graph.replay()
        with torch.cuda.stream(side):
            eager = step(x, dh)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want)) and all(torch.equal(a, b) for a, b in zip(eager, want))


def test_streams():
    """Two streams at once, and memory that is dropped before a side stream has used it."""
    step = _block(128, 300)
    x, dh = _normal(400, 128, seed=7, dtype=torch.bfloat16), _normal(400, 128, seed=8, dtype=torch.bfloat16)
    want = step(x, dh)
    torch.cuda.synchronize()
    sides = [torch.cuda.Stream() for _ in range(3)]
    results = []
    for _ in range(4):
        for s in sides:
            s.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(s):
                results.append(step(x, dh))
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for r in results for a, b in zip(r, want))
    # a layer and a joint made and run forward here, backward on a side stream that is late, and dropped at once
    w, pw = _normal(512, 512, seed=9, dtype=torch.float32), torch.ones(512, device="cuda")
    x, dy = _normal(700, 512, seed=10, dtype=torch.bfloat16), _normal(700, 512, seed=11, dtype=torch.bfloat16)

    def make():
        layer, joint = Linear16(w, activation="gelu"), ResidualNorm("rms", post_weight=pw.clone(), p=0.1)
        layer.forward(x, training=True)
        joint.forward(x.clone(), training=True)
        return layer, joint
    layer, joint = make()
    ref = [*layer.backward(dy)[:2], joint.backward(dy)[0]]
    for _ in range(3):
        layer, joint = make()
        side = sides[0]
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            torch.cuda._sleep(20_000_000)
        got = [*layer.backward(dy, stream=side)[:2], joint.backward(dy, stream=side)[0]]
        del layer, joint
        junk = [torch.full((700, 512), float("nan"), dtype=torch.bfloat16, device="cuda") for _ in range(20)]      # takes what was given back
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, ref))
        del junk
    # kept here, used on the side stream for something else in between: what was kept is this stream's all the same
    want = ref[2]
    for _ in range(3):
        _, joint = make()
        side.wait_stream(torch.cuda.current_stream())
        joint.forward(dy, stream=side)
        with torch.cuda.stream(side):
            torch.cuda._sleep(20_000_000)
        got = joint.backward(dy, stream=side)[0]
        del joint
        junk = [torch.full((700, 512), float("nan"), dtype=torch.bfloat16, device="cuda") for _ in range(20)]
        torch.cuda.synchronize()
        assert torch.equal(got, want)
        del junk
    for stream in (None, sides[1]):
        y = linear16(x, w.to(torch.bfloat16), stream=stream)
        z = dropout(x, 0.5, 1, stream=stream)
        torch.cuda.synchronize()
        assert torch.equal(y, linear16(x, w.to(torch.bfloat16))) and torch.equal(z, dropout(x, 0.5, 1))


def test_more_than_2_31_entries():
    """Offsets beyond 32 bits: the last rows as a call on them alone gives them."""
    rows, cols = 70_000, 32_768
    x = torch.empty(rows, cols, dtype=torch.bfloat16, device="cuda").fill_(0.5)
    x[-40:] = _normal(40, cols, seed=1, dtype=torch.bfloat16)
    tail = x[-40:].clone()
    w = 1 + _normal(cols, seed=2, scale=0.1)
    op = ResidualNorm("rms", pre_weight=w)
    h, n = op.forward(x, x, training=True)
    small = ResidualNorm("rms", pre_weight=w)
    hs, ns = small.forward(tail, tail, training=True)
    assert torch.equal(h[-40:], hs) and torch.equal(n[-40:], ns)
    del h
    dy, dx, _ = op.backward(n, x)
    sy, sx, _ = small.backward(ns, tail)
    assert torch.equal(dy[-40:], sy) and torch.equal(dx[-40:], sx)
    del dy, dx, n, op
    y = dropout(x, 0.5, 3)
    ones = torch.ones(rows, 8, dtype=torch.bfloat16, device="cuda")
    mask = dropout(ones, 0.5, 3)[-40:] != 0                 # the same counters in the first eight columns
    assert torch.equal(y[-40:, :8] != 0, mask & (tail[:, :8] != 0))
    del y
    wide = _normal(64, cols, seed=4, dtype=torch.bfloat16, scale=0.01)
    out = linear16(x, wide, activation="silu")
    # the same sums in another order: within the roundings of 32768 additions and half a step
    off = cols * 2.0 ** -23 * (tail.double().abs() @ wide.double().abs().T)
    z = tail.double() @ wide.double().T
    assert bool(((out[-40:].double() - torch.nn.functional.silu(z)).abs() <= 2.0 ** -8 * z.abs() + 1.1 * off).all())
    del out
    tall = torch.ones(rows, 16, dtype=torch.bfloat16, device="cuda")
    tall[-1] = 3
    out = linear16(tall, torch.ones(cols, 16, dtype=torch.bfloat16, device="cuda"))
    assert bool((out[-1] == 48).all()) and bool((out[-2] == 16).all()) and bool((out[0] == 16).all()) and bool((out[rows // 2] == 16).all())


@pytest.mark.parametrize("odd", [0, 1])
@pytest.mark.parametrize("m", [1, 8, 9, 16, 17, 32])
@pytest.mark.parametrize("k,n", [(64, 300), (520, 4736), (512, 4752), (264, 7104), (520, 7120), (1032, 9472), (512, 9504), (256, 11008), (2056, 640), (2048, 2048), (1024, 4096), (8200, 2368),
                                 (8200, 2384), (16400, 136)])
def test_few_tokens_by_every_form(m, k, n, odd):
    """Sizes on either side of where another form takes over on 148 SMs; tokens on 16-byte boundaries and not.  Whole numbers: exact."""
    gen = torch.Generator(device="cuda").manual_seed(m + n)
    x, w = (torch.randint(-2, 3, s, device="cuda", generator=gen).to(torch.bfloat16) for s in ((m, k + odd), (n, k)))
    x, b = x[:, odd:], torch.randint(-9, 10, (n,), device="cuda", generator=gen).float()
    z = x.double() @ w.double().T + b
    assert torch.equal(linear16(x, w, b, "relu", out_dtype=torch.float32), torch.relu(z).float())
    layer = Linear16(w, b, "relu")
    assert torch.equal(layer.forward(x, training=True), torch.relu(z).to(torch.bfloat16))
    dy = torch.randint(-2, 3, (m, n), device="cuda", generator=gen).to(torch.bfloat16)
    assert torch.equal(layer.backward(dy, grad_dtype=torch.float32, need_dx=False)[2], (dy.double() * (z > 0)).sum(0).float())

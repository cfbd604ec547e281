"""The first calls of a process captured into a graph."""
import pytest
import torch

from paper_1905_05957_b200 import Int8Linear, Int8Matrix, int8_linear, int8_matmul, int8_quantize, matrix_ops

pytestmark = pytest.mark.gpu


def _randn(*shape, seed):
    return torch.randn(*shape, device="cuda", generator=torch.Generator(device="cuda").manual_seed(seed))


@pytest.mark.parametrize("m", [1, 40, 300])
def test_products_captured_before_any_other(m, monkeypatch):
    x, w = _randn(m, 512, seed=m), int8_quantize(_randn(256, 512, seed=2))
    w = Int8Matrix.pack(w.codes, w.scale)
    want = int8_linear(x, w)
    y, z = torch.empty_like(want), torch.empty_like(want)
    torch.cuda.synchronize()
    monkeypatch.setattr(matrix_ops, "_status", {})      # as a process starts
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        int8_linear(x, w, out=y)
        int8_matmul(int8_quantize(x), w, out=z)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(y, want) and torch.equal(z, want)
    int8_matmul(int8_quantize(x), w)                    # outside: the status word is made
    assert matrix_ops.device_status() == 0 and matrix_ops._status


def test_a_training_step_captured_before_any_other(monkeypatch):
    x, w, dy = _randn(300, 512, seed=1), _randn(256, 512, seed=2), _randn(300, 256, seed=3)

    def step():
        layer = Int8Linear(w, torch.zeros(256, device="cuda"))
        return layer.forward(x, training=True), *layer.backward(dy)

    want = step()
    torch.cuda.synchronize()
    monkeypatch.setattr(matrix_ops, "_status", {})
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step()
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))

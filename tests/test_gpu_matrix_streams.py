"""Memory that the matrix operators own and streams other than the one it was allocated on: what is dropped before the stream has run may
not be handed out again until it has."""
import pytest
import torch

from paper_1905_05957_b200 import Int8Linear, Int8Matrix, OrthUpdate, int8_linear, int8_matmul, int8_quantize, matrix_ops
from paper_1905_05957_b200.matrix_ops import device_status

pytestmark = pytest.mark.gpu


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _behind():
    """A stream with some milliseconds of work before whatever comes next."""
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        busy = torch.randn(4096, 4096, device="cuda")
        for _ in range(40):
            busy = torch.sin(busy)
    return s


def _overwrite(sizes):
    """Allocations of these many bytes on the current stream, filled with what would be NaN in any type."""
    for _ in range(4):
        held = [torch.full((n,), 0xFF, dtype=torch.uint8, device="cuda") for n in sizes]
        del held


@pytest.mark.parametrize("m,n", [(300, 500), (1000, 512), (40, 72)])
def test_a_plan_dropped_before_its_stream_has_run(m, n):
    g = torch.randn(m, n, device="cuda", generator=_gen(m))
    buf0 = torch.randn(m, n, device="cuda", generator=_gen(n))
    keep = OrthUpdate(m, n)
    want_buf, x0 = buf0.clone(), torch.randn(m, n, device="cuda", generator=_gen(3))
    want_x = x0.clone()
    want = keep.update(g, want_buf, out_dtype=torch.float32, x=want_x, gamma=0.1)
    sizes = (keep.workspace.numel(), keep.workspace.numel() // 2, 512, 16)
    buf, x, out = buf0.clone(), x0.clone(), torch.empty(m, n, device="cuda")
    torch.cuda.synchronize()
    plan = OrthUpdate(m, n)
    s = _behind()
    plan.update(g, buf, out=out, x=x, gamma=0.1, stream=s)
    del plan
    _overwrite(sizes)
    torch.cuda.synchronize()
    assert torch.equal(out, want[0]) and torch.equal(buf, want_buf) and torch.equal(x, want_x)


def _weights(n, k, seed):
    return torch.randn(n, k, device="cuda", generator=_gen(seed))


@pytest.mark.parametrize("m", [1, 40, 300])
@pytest.mark.parametrize("made", ["quantised", "packed"])
def test_codes_dropped_before_their_stream_has_run(m, made):
    """Weights and tokens quantised on the current stream, used on another and dropped."""
    x, w = _weights(m, 512, 1), _weights(256, 512, 2)

    def make(v):
        q = int8_quantize(v)
        return Int8Matrix.pack(q.codes, q.scale) if made == "packed" else q

    want = int8_linear(x, make(w)), int8_matmul(make(x), make(w))
    y, z = torch.empty_like(want[0]), torch.empty_like(want[1])
    torch.cuda.synchronize()
    a, b, c = make(x), make(w), make(w)
    s = _behind()
    int8_linear(x, b, out=y, stream=s)
    int8_matmul(a, c, out=z, stream=s)
    del a, b, c
    _overwrite([256 * 512 + 4 * 256 + 16, 256 * 512, 4 * 256, m * 512 + 4 * 304 + 16, m * 512, 4 * m, 16])
    torch.cuda.synchronize()
    assert torch.equal(y, want[0]) and torch.equal(z, want[1])


def test_a_layer_dropped_before_its_stream_has_run():
    x, w, dy = _weights(300, 512, 1), _weights(256, 512, 2), _weights(300, 256, 3)
    layer = Int8Linear(w)
    layer.forward(x, training=True)
    want = layer.backward(dy)[1]
    dw = torch.empty_like(want)
    layer.forward(x, training=True)      # codes of x and W on the current stream, the backward pass on another
    torch.cuda.synchronize()
    s = _behind()
    layer.backward(dy, dw=dw, stream=s)
    del layer
    _overwrite([300 * 512 + 512 * 304 + 4 * 816 + 16, 256 * 512 * 2 + 4 * 768 + 16, 300 * 512, 256 * 512])
    torch.cuda.synchronize()
    assert torch.equal(dw, want)


def test_status_of_products_on_other_streams():
    """What a product on a stream that is behind reports is seen: here the words are set as such a product would set them."""
    plan = OrthUpdate(8, 16)
    assert device_status() == 0 and not plan.timed_out()
    word = matrix_ops._status[torch.cuda.current_device()][0]
    s = _behind()
    with torch.cuda.stream(s):
        word.fill_(2)
        plan.dev_status[:1].fill_(2)
    seen = device_status(), plan.timed_out()
    torch.cuda.synchronize()
    word.zero_()
    assert seen == (2, True)
    s = _behind()
    with torch.cuda.stream(s):
        plan.dev_status[:1].fill_(0)
    assert not plan.timed_out() and device_status() == 0

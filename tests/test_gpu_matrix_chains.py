"""Chains of calls in which each reads what the one before wrote, at addresses that are written anew every round: launches wait for one another
while already resident, so nothing may be read that was fetched before the wait."""
import pytest
import torch

from paper_1905_05957_b200 import Int8Matrix, OrthUpdate, int8_linear, int8_matmul, int8_quantize

pytestmark = pytest.mark.gpu


def _randn(*shape, seed):
    return torch.randn(*shape, device="cuda", generator=torch.Generator(device="cuda").manual_seed(seed))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("m", [1, 7, 16, 40, 200])
def test_layers_one_after_another(m, dtype):
    """y1 = x W1^T, y2 = y1 W2^T, x = y2: three buffers, twelve rounds, without a wait between the launches."""
    w1, w2 = (int8_quantize(_randn(512, 512, seed=s) / 512 ** 0.5) for s in (1, 2))
    x0 = _randn(m, 512, seed=m).to(dtype)
    want, v = [], x0
    for _ in range(12):
        u = int8_linear(v, w1)
        torch.cuda.synchronize()
        v = int8_linear(u, w2)
        torch.cuda.synchronize()
        want.append(v)
    for _ in range(5):
        x, y = x0.clone(), torch.empty_like(x0)
        got = torch.empty(12, m, 512, dtype=dtype, device="cuda")
        torch.cuda.synchronize()
        for i in range(12):
            int8_linear(x, w1, out=y)
            int8_linear(y, w2, out=x)
            got[i].copy_(x)
        assert torch.equal(got, torch.stack(want))
        x.copy_(x0)
        for _ in range(12):                  # and with nothing between them but the calls
            int8_linear(x, w1, out=y)
            int8_linear(y, w2, out=x)
        assert torch.equal(x, want[-1])


@pytest.mark.parametrize("m", [1, 16, 100])
def test_weights_written_by_the_launch_before(m):
    """Weights, scales and bias change in place right before the call that reads them."""
    made = [int8_quantize(_randn(384, 640, seed=10 + i)) for i in range(4)]
    biases = [_randn(384, seed=20 + i) for i in range(4)]
    x = _randn(m, 640, seed=5)
    want = [int8_linear(x, w, b) for w, b in zip(made, biases)]
    torch.cuda.synchronize()
    w = Int8Matrix(torch.empty_like(made[0].codes.contiguous()), torch.empty(384, device="cuda"))
    bias = torch.empty(384, device="cuda")
    for _ in range(10):
        got = []
        for v, b in zip(made, biases):
            w.codes.copy_(v.codes)
            w.scale.copy_(v.scale)
            bias.copy_(b)
            got.append(int8_linear(x, w, bias))
        assert all(torch.equal(a, b) for a, b in zip(got, want))


@pytest.mark.parametrize("m,n", [(40, 72), (130, 261), (300, 500)])
def test_quantise_multiply_and_update_in_a_row(m, n):
    """dW = dY^T x straight into the update of W, whose new values are quantised for the next round."""
    def run(wait):
        x, dy, w = _randn(64, n, seed=1), _randn(64, m, seed=2), _randn(m, n, seed=3)
        plan, buf, g = OrthUpdate(m, n), torch.zeros(m, n, device="cuda"), torch.empty(m, n, device="cuda")
        out = []
        for _ in range(8):
            q = int8_quantize(w)
            wait()
            y = int8_linear(x, q, out_dtype=torch.float32)
            wait()
            dc = int8_quantize(dy + 0.01 * y, rows=False, cols=True)
            wait()
            int8_matmul(dc, int8_quantize(x, rows=False, cols=True), out=g)
            wait()
            plan.update(g, buf, out_dtype=None, x=w, gamma=0.1)
            wait()
            out.append(w.clone())
        return out
    want = run(torch.cuda.synchronize)
    for _ in range(5):
        assert all(torch.equal(a, b) for a, b in zip(run(lambda: None), want))


@pytest.mark.parametrize("m", [1, 16, 100])
def test_an_output_over_its_input_is_refused(m):
    w = int8_quantize(_randn(256, 256, seed=1))
    store = torch.zeros(2 * m + 1, 256, device="cuda")
    x = store[:m]
    for out in (x, store[m - 1:2 * m - 1], x.view(torch.bfloat16)[:, :256]):
        with pytest.raises(ValueError, match="overlap"):
            int8_linear(x, w, out=out)
    x.copy_(_randn(m, 256, seed=2))
    assert torch.equal(int8_linear(x, w, out=store[m:2 * m]), int8_linear(x, w))          # right behind it is not over it
    assert (store[2 * m:] == 0).all()

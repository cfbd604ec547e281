"""Memory that layers and joints use without owning it: parameters whose storage is replaced between calls, and tensors that belong to another stream than the one that uses them."""
import ctypes as C
import os
import subprocess
import sys

import pytest
import torch

from paper_1905_05957_b200 import DsqError, Linear16, ResidualNorm, binding, linear16

pytestmark = pytest.mark.gpu


def _normal(*shape, seed, dtype=torch.float32, scale=1.0):
    return (scale * torch.randn(*shape, device="cuda", generator=torch.Generator(device="cuda").manual_seed(seed))).to(dtype)


@pytest.mark.parametrize("groups", [0, 3])
def test_a_joint_whose_parameters_get_other_storage(groups):
    rows, cols = 12, 200
    shapes = {"post_weight": (cols,), "post_bias": (cols,), "gate": (groups, cols) if groups else (cols,), "pre_weight": (cols,), "pre_bias": (cols,)}
    params = {k: _normal(*s, seed=i) for i, (k, s) in enumerate(shapes.items())}
    op = ResidualNorm("layer", **params)
    y, x, dh, dn = (_normal(rows, cols, seed=20 + i) for i in range(4))
    op.forward(y, x, training=True)
    op.backward(dh, dn)
    for i, (k, s) in enumerate(shapes.items()):
        if i % 2:
            params[k].data = _normal(*s, seed=40 + i)
        else:
            params[k].set_(_normal(*s, seed=40 + i))
    junk = [torch.full((4096,), float("nan"), device="cuda") for _ in range(64)]      # takes what was given back
    got = [*op.forward(y, x, training=True), *op.backward(dh, dn)[:2]]
    grads = op.backward(dh, dn)[2]
    other = ResidualNorm("layer", **{k: v.clone() for k, v in params.items()})
    want = [*other.forward(y, x, training=True), *other.backward(dh, dn)[:2]]
    assert all(torch.equal(a, b) for a, b in zip(got, want)) and all(torch.equal(grads[k], v) for k, v in other.backward(dh, dn)[2].items())
    del junk
    params["pre_weight"].data = params["pre_weight"].data[:cols - 8]
    with pytest.raises(ValueError):
        op.forward(y, x)
    with pytest.raises(ValueError):
        op.backward(dh, dn)


@pytest.mark.parametrize("dropped", ["object", "next forward"])
def test_tensors_of_another_stream(dropped):
    """Weights, parameters and inputs that belong to the main stream, all used on a late side stream alone, then dropped here: what is allocated here next must not be theirs."""
    rows, width = 600, 512
    x, dy = _normal(rows, width, seed=1, dtype=torch.bfloat16), _normal(rows, width, seed=2, dtype=torch.bfloat16)
    w, v = _normal(width, width, seed=3, dtype=torch.bfloat16, scale=width ** -0.5), 1 + _normal(width, seed=4, scale=0.1)

    def make(stream):
        with torch.cuda.stream(torch.cuda.current_stream() if stream is None else stream):
            layer, joint = Linear16(own[0], own[1], "gelu"), ResidualNorm("layer", post_weight=own[2], pre_weight=own[3])
            return layer, joint, layer.forward(own[4], training=True), *joint.forward(own[5], own[6], training=True)

    def copies():
        return [t.clone() for t in (w, v, v, v, x, x, dy)]
    own = copies()
    layer, joint, *want = make(None)
    want += [*layer.backward(dy), *joint.backward(dy, dy)[:2]]
    side = torch.cuda.Stream()
    for _ in range(3):
        own = copies()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            torch.cuda._sleep(20_000_000)
        layer, joint, *got = make(side)
        with torch.cuda.stream(side):
            got += [*layer.backward(dy), *joint.backward(dy, dy)[:2]]
            if dropped == "next forward":
                layer.forward(x, training=True)
                joint.forward(x, dy, training=True)
        del own
        if dropped == "object":
            del layer, joint
        junk = [torch.full((rows, width), float("nan"), dtype=torch.bfloat16, device="cuda") for _ in range(20)]
        junk += [torch.full((width,), float("nan"), device="cuda") for _ in range(20)]
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))
        del junk


def test_single_rows_in_place_whatever_their_pitches():
    """Through the C ABI, which takes pitches that the Python calls work out: of one row they mean nothing."""
    lib = binding.load_library()
    x, w, r = (_normal(*s, seed=i, dtype=torch.bfloat16) for i, s in enumerate(((1, 64), (48, 64), (1, 48))))
    want, out = linear16(x, w, residual=r), r.clone()
    p = binding.ds_f16_product(dtype=binding.DS_BF16, m=1, n=48, k=64, a=x.data_ptr(), lda=3, b=w.data_ptr(), ldb=64, residual=out.data_ptr(), ldr=5, out=out.data_ptr(),
                               out_dtype=binding.DS_BF16, ldo=9)
    stream = torch.cuda.current_stream().cuda_stream
    assert lib.ds_f16_matmul(C.byref(p), stream) == binding.DS_OK
    assert torch.equal(out, want)
    dy, z = _normal(1, 48, seed=3, dtype=torch.bfloat16), _normal(1, 48, seed=4, dtype=torch.bfloat16)
    want = torch.where(z > 0, dy, torch.zeros_like(dy))
    for over in (dy.clone(), z.clone()):
        given = [over if torch.equal(over, t) else t for t in (dy, z)]
        p = binding.ds_f16_slope_args(dtype=binding.DS_BF16, rows=1, cols=48, dy=given[0].data_ptr(), lddy=2, z=given[1].data_ptr(), ldz=3, activation=1, dz=over.data_ptr(), lddz=5)
        assert lib.ds_f16_slope(C.byref(p), stream) == binding.DS_OK
        assert torch.equal(over, want)


def test_parameters_between_wider_rows():
    """A vector in the columns that the rows of an output leave free shares no memory with it; one in its rows does."""
    rows, cols = 9, 64
    buf = torch.zeros(rows, 2 * cols, device="cuda")
    h, w = buf[:, :cols], buf[3, cols:]
    w.copy_(1 + _normal(cols, seed=1))
    y, x = _normal(rows, cols, seed=2), _normal(rows, cols, seed=3)
    want = ResidualNorm("layer", post_weight=w.clone()).forward(y, x)[0]
    op = ResidualNorm("layer", post_weight=w)
    op.forward(y, x, h=h)
    assert torch.equal(h, want)
    for at in (0, 5, cols - 1):
        with pytest.raises(DsqError):
            ResidualNorm("layer", post_weight=buf[3, at:at + cols]).forward(y, x, h=h)


def test_as_many_tokens_as_a_layer_trains_on():
    """Whole numbers whose sums are exact."""
    m = 2097120
    x, w = torch.ones(m, 8, dtype=torch.bfloat16, device="cuda"), torch.ones(16, 8, dtype=torch.bfloat16, device="cuda")
    x[-1] = 2
    layer = Linear16(w, torch.zeros(16, device="cuda"), "relu")
    assert bool((layer.forward(x, training=True)[-1] == 16).all())
    dx, dw, db = layer.backward(x.repeat(1, 2), grad_dtype=torch.float32)
    assert bool((dx[:-1] == 16).all()) and bool((dx[-1] == 32).all()) and bool((dw == m - 1 + 4).all()) and bool((db == m - 1 + 2).all())
    with pytest.raises(ValueError):
        layer.forward(torch.ones(m + 1, 8, dtype=torch.bfloat16, device="cuda"), training=True)


FIRST = """
import sys
import torch
from paper_1905_05957_b200 import ResidualNorm, linear16
x, w = (torch.ones(s, 2048, device="cuda", dtype=torch.bfloat16) for s in (int(sys.argv[1]), 6144))
norm = torch.ones(2048, device="cuda")
torch.cuda.synchronize()
graph = torch.cuda.CUDAGraph()
with torch.cuda.graph(graph):
    y = linear16(x, w)
    n = ResidualNorm("rms", pre_weight=norm).forward(x)[1]
y.zero_()
graph.replay()
torch.cuda.synchronize()
assert bool((y == 2048).all()) and bool((n == 1).all())
"""


@pytest.mark.parametrize("tokens", [1, 12])
def test_a_process_whose_first_call_is_captured(tokens):
    """What is asked of the device once, how many CTAs an SM holds among it, may be asked while a graph is captured."""
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    subprocess.run([sys.executable, "-c", FIRST, str(tokens)], cwd=root, check=True, timeout=300)

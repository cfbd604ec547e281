"""What the layers and joints hand to the library and tell the allocator, on a host without a device: tensors that have an address, a type and a place but no memory,
and calls that are noted instead of made."""
import types

import pytest
import torch

from paper_1905_05957_b200 import Int8Linear, Int8Matrix, int8_matmul, layer_ops, matrix_ops
from paper_1905_05957_b200.layer_ops import Linear16, ResidualNorm

F32, BF16 = torch.float32, torch.bfloat16


class Tensor:
    """Rows of consecutive entries at an address of their own."""
    last = 0x10000

    def __init__(self, *shape, dtype=F32, index=0, owner="caller"):
        self.shape, self.dtype, self.index, self.owner = torch.Size(shape), dtype, index, owner
        self.used_on = set()
        self.renew()

    def renew(self):
        """Other storage for the same tensor."""
        Tensor.last += 1 << 24
        self.address, self.used_on = Tensor.last, set()

    device = property(lambda self: torch.device("cuda", self.index) if self.index >= 0 else torch.device("cpu"))
    is_cuda = property(lambda self: self.index >= 0)

    def dim(self):
        return len(self.shape)

    def numel(self):
        return self.shape.numel()

    def stride(self):
        return tuple(self.shape[i + 1:].numel() for i in range(len(self.shape)))

    def get_device(self):
        return self.index

    def is_contiguous(self):
        return True

    def contiguous(self):
        return self

    def data_ptr(self):
        return self.address

    def detach(self):
        view = Tensor(*self.shape, dtype=self.dtype, index=self.index, owner=self.owner)
        view.address, view.used_on = self.address, self.used_on      # one storage
        return view

    def new_empty(self, shape, dtype=None):
        return Tensor(*((shape,) if isinstance(shape, int) else shape), dtype=dtype or self.dtype, index=self.index, owner="package")

    def record_stream(self, stream):
        if self.index < 0:
            raise NotImplementedError("record_stream on the host")
        self.used_on.add(stream.name)


@pytest.fixture
def host(monkeypatch):
    """.calls: (address of the function, stream, members...);  .on(stream): what follows runs there."""
    h = types.SimpleNamespace(calls=[], stream=0)

    def note(where, stream, *members):
        h.calls.append((where, stream, members))
        return 0

    def note_call(where, *args):
        h.calls.append((where, args[-1], args[:-1]))
        return 0
    for name, value in dict(_struct=note, _call=note_call, _size=lambda *a: 0, _slope_ws=lambda r, c: 0, _raw_stream=lambda index: h.stream, _current=lambda: 0,
                            _status={0: (None, 0)}, _matmul_at="matmul", _slope_at="slope", _pack_at="pack", _norm_at="forward", _norm_back_at="backward",
                            _like_of=lambda t: Tensor(*t.shape, dtype=t.dtype, index=t.index, owner="package")).items():
        monkeypatch.setattr(layer_ops, name, value)
    for name, value in dict(_call=note_call, _linear_ws=lambda *a: 0, _quantize_ws=lambda *a: 0, _raw_stream=lambda index: h.stream, _current=lambda: 0, _status={0: (None, 0)}, _streams={},
                            _linear_at="linear", _quantize_at="quantize", _matmul_at="matmul",
                            _empty=lambda *shape, dtype, device: Tensor(*(shape[0] if isinstance(shape[0], tuple) else shape), dtype=dtype, owner="package")).items():
        monkeypatch.setattr(matrix_ops, name, value, raising=name != "_streams")
    monkeypatch.setattr(torch.cuda, "current_stream", lambda index=None: types.SimpleNamespace(name=h.stream, cuda_stream=h.stream))

    def on(stream):
        h.stream = stream
    h.on = on
    return h


def _addresses(call):
    return [m for m in call[2] if isinstance(m, int) and m > 1 << 24]


PARAMETERS = ("post_weight", "post_bias", "gate", "pre_weight", "pre_bias")


@pytest.mark.parametrize("name", PARAMETERS)
def test_a_joint_reads_a_parameter_where_it_is_now(host, name):
    params = {k: Tensor(64) for k in PARAMETERS}
    op, y, x = ResidualNorm("layer", **params), Tensor(6, 64), Tensor(6, 64)
    old = params[name].address
    op.forward(y, x, training=True)
    op.backward(x)
    assert all(old in _addresses(c) for c in host.calls)
    params[name].renew()
    del host.calls[:]
    op.forward(y, x, training=True)
    op.backward(x)
    assert len(host.calls) == 2
    assert all(old not in _addresses(c) and params[name].address in _addresses(c) for c in host.calls)


@pytest.mark.parametrize("name", PARAMETERS)
@pytest.mark.parametrize("change", [dict(shape=torch.Size((60,))), dict(dtype=BF16), dict(index=1)], ids=str)
def test_a_joint_refuses_a_parameter_that_no_longer_fits(host, name, change):
    """Its kernels would read, and write gradients, past what is there."""
    params = {k: Tensor(64) for k in PARAMETERS}
    op, y = ResidualNorm("layer", **params), Tensor(6, 64)
    op.forward(y, training=True)
    for k, v in change.items():
        setattr(params[name], k, v)
    del host.calls[:]
    with pytest.raises(ValueError):
        op.forward(y)
    with pytest.raises(ValueError):
        op.backward(y)
    assert not host.calls


def test_a_joint_counts_the_gates_that_are_there(host):
    gate = Tensor(2, 64)
    op, y = ResidualNorm("rms", gate=gate), Tensor(6, 64)
    op.forward(y, training=True)
    gate.shape = torch.Size((4, 64))
    with pytest.raises(ValueError):
        op.forward(y)                       # six rows are not four runs
    with pytest.raises(ValueError):
        op.backward(y)
    gate.shape = torch.Size((3, 64))
    del host.calls[:]
    op.forward(y)
    assert 3 in host.calls[0][2]


def test_a_layer_keeps_the_weights_that_it_was_given(host):
    """Until set_weight(): a tensor that has other memory or another shape since then is not read by the sizes that it had."""
    w, x = Tensor(48, 64, dtype=BF16), Tensor(100, 64, dtype=BF16)
    layer, old = Linear16(w), w.address
    w.renew()
    w.shape, w.index = torch.Size((10, 64)), 1
    layer.forward(x, training=True)
    layer.backward(Tensor(100, 48, dtype=BF16))
    assert all(w.address not in _addresses(c) for c in host.calls) and old in _addresses(host.calls[0])
    w.index = 0
    layer.set_weight(w)
    del host.calls[:]
    assert layer.forward(x).shape == (100, 10) and w.address in _addresses(host.calls[0])


@pytest.mark.parametrize("change", [dict(shape=torch.Size((1, 8))), dict(shape=torch.Size((100, 60))), dict(dtype=torch.float16), dict()], ids=str)
@pytest.mark.parametrize("which", ["x", "y", "r"])
def test_backward_reads_what_forward_read(host, which, change):
    """Inputs that have other memory, sizes or types since then are refused."""
    layer, op = Linear16(Tensor(48, 64, dtype=BF16)), ResidualNorm("rms", pre_weight=Tensor(64))
    given = dict(x=Tensor(100, 64, dtype=BF16), y=Tensor(100, 64, dtype=BF16), r=Tensor(100, 64))
    layer.forward(given["x"], training=True)
    op.forward(given["y"], given["r"], training=True)
    layer.backward(Tensor(100, 48, dtype=BF16))
    op.backward(Tensor(100, 64))
    del host.calls[:]
    for k, v in change.items():
        setattr(given[which], k, v)
    if not change:
        given[which].renew()
    with pytest.raises(RuntimeError):
        layer.backward(Tensor(100, 48, dtype=BF16)) if which == "x" else op.backward(Tensor(100, 64))
    assert not host.calls


def test_the_allocator_is_told_where_a_layer_uses_what_it_was_given(host):
    """Memory that belongs to another stream, used on one stream alone: the tensors may belong to any stream, so it is told of that one."""
    host.on(7)
    w, b, x = Tensor(48, 64, dtype=BF16), Tensor(48), Tensor(100, 64, dtype=BF16)
    layer = Linear16(w, b, "gelu")
    layer.forward(x, training=True)
    layer.backward(Tensor(100, 48, dtype=BF16))
    assert w.used_on == b.used_on == x.used_on == {7}
    layer.bias = other = Tensor(48)
    layer.forward(x)
    other.renew()                                 # other storage, the stream of the last call
    layer.forward(x)
    assert other.used_on == {7}
    host.on(8)
    layer.forward(x)
    assert w.used_on == other.used_on == {7, 8} and x.used_on == {7}      # x: no training, the caller's alone
    layer.backward(Tensor(100, 48, dtype=BF16))
    assert x.used_on == layer._z.used_on | {7} == {7, 8}
    host.on(9)
    layer = Linear16(w, b)
    layer.forward(x)
    layer.set_weight(Tensor(48, 64, dtype=BF16))
    assert w.used_on == {7, 8, 9} and b.used_on == {7, 9}
    layer.bias.index = -1                         # on the host: refused as ever
    with pytest.raises(ValueError):
        layer.forward(x)


def test_the_allocator_is_told_where_a_joint_uses_what_it_was_given(host):
    host.on(7)
    params = {k: Tensor(64) for k in PARAMETERS}
    op, y, x = ResidualNorm("layer", **params), Tensor(6, 64), Tensor(6, 64)
    op.forward(y, x)
    assert all(t.used_on == {7} for t in params.values()) and not y.used_on and not x.used_on
    op.forward(y, x, training=True)
    assert y.used_on == x.used_on == {7}
    host.on(8)
    op.backward(x)
    assert all(t.used_on == {7, 8} for t in (y, x, *params.values())) and op._saved[4].used_on == {8}
    for t in params.values():
        t.renew()                                 # other storage, the stream of the last call
    op.backward(x)
    assert all(t.used_on == {8} for t in params.values())
    host.on(7)
    op.forward(y, x)
    assert all(t.used_on == {7, 8} for t in params.values())


def test_more_tokens_than_backward_takes_are_refused_forward(host):
    """2097120, where the column sums and slopes are taken; nothing is launched."""
    w, b = Tensor(16, 8, dtype=BF16), Tensor(16)
    x = Tensor(2097121, 8, dtype=BF16)
    for layer in (Linear16(w, b), Linear16(w, activation="relu")):
        with pytest.raises(ValueError):
            layer.forward(x, training=True)
        assert not host.calls
        layer.forward(x)
        layer.forward(Tensor(2097120, 8, dtype=BF16), training=True)
        del host.calls[:]
    Linear16(w).forward(x, training=True)


def test_the_allocator_is_told_where_8_bit_matrices_and_biases_are_used(host):
    """As above; codes that the package made belong to the stream that made them."""
    host.on(7)
    codes, scale = Tensor(32, 64, dtype=torch.int8), Tensor(32)
    m = Int8Matrix(codes, scale)
    int8_matmul(m, m)
    assert codes.used_on == scale.used_on == {7}
    host.on(8)
    int8_matmul(m, m)
    assert codes.used_on == scale.used_on == {7, 8}
    b, other, x = Tensor(48), Tensor(48), Tensor(16, 64, dtype=BF16)
    layer = Int8Linear(Tensor(48, 64), b)
    layer.forward(x)
    host.on(9)
    layer.forward(x, training=True)
    assert layer.by_rows._codes[0].used_on == {9}
    layer.bias = other
    layer.forward(x)
    other.renew()                                 # other storage, the stream of the last call
    layer.forward(x)
    assert b.used_on == {8, 9} and other.used_on == {9}
    other.index = -1                              # on the host: refused as ever
    for training in (False, True):
        with pytest.raises(ValueError):
            layer.forward(x, training=training)

"""The 16-bit layer against arithmetic in 64 bits.

Whole numbers whose sums stay below 2^24 are summed exactly in 32 bits in any order, so that products without an activation have one right answer: the exact sum,
rounded once.  Elsewhere the tolerances are bounds: half a step of the result's type, K roundings of 2^-23 of the sum of magnitudes, 2^-20 for the activations'
functions (a few units of 2^-22 each), carried through what follows.
"""
import pytest
import torch

from paper_1905_05957_b200 import DsqError, Linear16, linear16

pytestmark = pytest.mark.gpu
HALVES = [torch.bfloat16, torch.float16]
ACTS = {"none": lambda z: z, "relu": torch.relu, "gelu": torch.nn.functional.gelu, "silu": torch.nn.functional.silu,
        "gelu_tanh": lambda z: torch.nn.functional.gelu(z, approximate="tanh")}


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _whole(shape, seed, dtype, most=3):
    return torch.randint(-most, most + 1, shape, device="cuda", generator=_gen(seed)).to(dtype)


def _normal(shape, seed, dtype, scale=1.0):
    return (scale * torch.randn(shape, device="cuda", generator=_gen(seed))).to(dtype)


SIZES = [(1, 1, 1), (1, 5, 3), (1, 64, 16), (1, 2048, 200), (3, 40, 70), (8, 129, 33), (9, 32, 64), (16, 1000, 100), (17, 64, 32), (20, 257, 129), (32, 512, 100),
         (33, 96, 520), (64, 128, 256), (65, 130, 258), (100, 8, 8), (128, 64, 64), (129, 72, 520), (333, 1000, 300), (257, 4096, 136), (700, 520, 1032), (2048, 512, 2048)]


@pytest.mark.parametrize("dtype", HALVES)
@pytest.mark.parametrize("m,k,n", SIZES)
def test_forward_of_whole_numbers_is_exact(m, k, n, dtype):
    x, w, r = _whole((m, k), 1, dtype), _whole((n, k), 2, dtype), _whole((m, n), 3, dtype, 100)
    b = _whole((n,), 4, torch.float32, 50)
    z = x.double() @ w.double().T
    assert float(z.abs().max()) + 150 < 2 ** 24
    assert torch.equal(linear16(x, w), z.to(dtype))
    assert torch.equal(linear16(x, w, out_dtype=torch.float32), z.float())
    assert torch.equal(linear16(x, w, b, "relu", r), (torch.relu(z + b) + r.double()).to(dtype))
    assert torch.equal(linear16(x, w, b, "none", r, out_dtype=torch.float32), (z + b + r.double()).float())
    y = r.clone()
    assert linear16(x, w, b, residual=y, out=y) is y and torch.equal(y, (z + b + r.double()).to(dtype))      # added to in place


@pytest.mark.parametrize("dtype", HALVES)
@pytest.mark.parametrize("m,k,n", SIZES)
def test_gradients_of_whole_numbers_are_exact(m, k, n, dtype):
    x, w, dy = _whole((m, k), 1, dtype), _whole((n, k), 2, dtype), _whole((m, n), 3, dtype)
    b = torch.zeros(n, device="cuda")
    layer = Linear16(w, b)
    layer.forward(x, training=True)
    x8, w8, d8 = x.double(), w.double(), dy.double()
    dx, dw, db = layer.backward(dy)
    assert torch.equal(dx, (d8 @ w8).to(dtype)) and torch.equal(dw, (d8.T @ x8).to(dtype)) and torch.equal(db, d8.sum(0).to(dtype))
    dx, dw, db = layer.backward(dy, grad_dtype=torch.float32, need_dx=False)
    assert dx is None and torch.equal(dw, (d8.T @ x8).float()) and torch.equal(db, d8.sum(0).float())


@pytest.mark.parametrize("m,k,n", [(1, 100, 70), (40, 100, 70), (300, 100, 70), (300, 96, 520)])
@pytest.mark.parametrize("pad,offset", [(0, 0), (8, 8), (3, 1), (16, 5)])
def test_rows_within_wider_rows(m, k, n, pad, offset):
    dtype = torch.bfloat16

    def within(t):
        r, c = t.shape
        buf = torch.full((offset + (r + 1) * (c + pad),), 7.0, dtype=t.dtype, device="cuda")
        v = buf[offset:offset + r * (c + pad)].view(r, c + pad)[:, :c] if pad or not offset else buf[offset:offset + r * c].view(r, c)
        v.copy_(t)
        return v, buf

    def stray(v, buf):
        """Whether anything but v was written in its buffer."""
        buf = buf.clone()
        buf.as_strided(v.shape, v.stride(), v.storage_offset()).fill_(7.0)
        return not bool((buf == 7.0).all())
    (x, _), (w, _), (r, _) = within(_whole((m, k), 1, dtype)), within(_whole((n, k), 2, dtype)), within(_whole((m, n), 3, dtype))
    z = x.double() @ w.double().T + r.double()
    for dt in (dtype, torch.float32):
        out, buf = within(torch.zeros(m, n, dtype=dt, device="cuda"))
        linear16(x, w, residual=r, out=out)
        assert torch.equal(out, z.to(dt)) and not stray(out, buf)
    layer = Linear16(w)
    y = layer.forward(x, residual=r, training=True)
    assert torch.equal(y, z.to(dtype))
    dy, _ = within(_whole((m, n), 4, dtype))
    dw, buf = within(torch.zeros(n, k, device="cuda"))
    dx, got, _ = layer.backward(dy, dw=dw)
    assert got is dw and torch.equal(dw, (dy.double().T @ x.double()).float()) and not stray(dw, buf)
    assert torch.equal(dx, (dy.double() @ w.double()).to(dtype))


@pytest.mark.parametrize("dtype", HALVES)
@pytest.mark.parametrize("m", [2, 12, 40, 100, 700])
@pytest.mark.parametrize("n", [1, 7, 31, 66, 129, 250, 255, 1001, 1004])
def test_rows_that_end_inside_16_bytes(m, n, dtype):
    """Operands and outputs whose rows start on 16-byte boundaries and end anywhere: what lies behind them is not read into sums (NaN) and not written."""
    def padded(*shape, fill=float("nan"), dt=dtype, seed=None):
        r, c = shape
        buf = torch.full((r, (c + 7) // 8 * 8 + 8), fill, dtype=dt, device="cuda")
        if seed is not None:
            buf[:, :c] = _whole(shape, seed, dt)
        return buf[:, :c], buf
    (x, _), (w, _), (r, _), (dy, _) = padded(m, 37, seed=1), padded(n, 37, seed=2), padded(m, n, seed=3), padded(m, n, seed=4)
    z = x.double() @ w.double().T
    for dt in (dtype, torch.float32):
        out, buf = padded(m, n, fill=7.0, dt=dt)
        linear16(x, w, residual=r, out=out)
        assert torch.equal(out, (z + r.double()).to(dt)) and bool((buf[:, n:] == 7.0).all())
    layer = Linear16(w, activation="relu")
    assert torch.equal(layer.forward(x, training=True), torch.relu(z).to(dtype))
    dz = dy.double() * (z > 0)
    for dt in (dtype, torch.float32):
        dw, buf = padded(n, 37, fill=7.0, dt=dt)
        dx, _, _ = layer.backward(dy, dw=dw)
        assert torch.equal(dx, (dz @ w.double()).to(dtype)) and torch.equal(dw, (dz.T @ x.double()).to(dt)) and bool((buf[:, 37:] == 7.0).all())
    layer = Linear16(dy.t().contiguous())          # gradients of weights whose rows end inside 16 bytes, on rows that do not
    layer.forward(r.t().contiguous()[:, :m], training=True)
    got, buf = padded(n, m, fill=7.0)
    layer.backward(_whole((n, n), 5, dtype), dw=got)
    assert bool((buf[:, m:] == 7.0).all())


def test_columns_of_one_buffer():
    buf = _whole((70, 96), 1, torch.bfloat16)
    x, w = buf[:, :32], _whole((64, 32), 2, torch.bfloat16)
    want = (x.double() @ w.double().T).to(torch.bfloat16)
    linear16(x, w, out=buf[:, 32:])
    assert torch.equal(buf[:, 32:], want)


@pytest.mark.parametrize("dtype", HALVES)
@pytest.mark.parametrize("act", list(ACTS))
@pytest.mark.parametrize("m,k,n", [(1, 300, 200), (13, 256, 72), (50, 64, 264), (333, 200, 136), (300, 128, 130)])
def test_activations_and_their_gradients(m, k, n, act, dtype):
    half = torch.finfo(dtype).eps / 2
    tiny = 2.0 ** -25 if dtype is torch.float16 else 0.0      # half a step among fp16's smallest numbers
    x, w, r, dy = _normal((m, k), 1, dtype, 2.0), _normal((n, k), 2, dtype, k ** -0.5), _normal((m, n), 3, dtype), _normal((m, n), 4, dtype)
    b = _normal((n,), 5, torch.float32)
    x8, w8, b8 = (t.double().requires_grad_() for t in (x, w, b))
    z = x8 @ w8.T + b8
    y = ACTS[act](z) + r.double()
    gx, gw, gb = torch.autograd.grad(y, (x8, w8, b8), dy.double())
    z, y = z.detach(), y.detach()
    sum_off = k * 2.0 ** -23 * (x.double().abs() @ w.double().abs().T + b.double().abs())
    layer = Linear16(w, b, act)
    for got in (linear16(x, w, b, act, r), layer.forward(x, residual=r, training=True)):
        off = (got.double() - y).abs()
        assert bool((off <= half * y.abs() + 1.13 * sum_off + 2.0 ** -20 * (z.abs() + y.abs()) + tiny).all())
    dx, dw, db = layer.backward(dy)
    # dz: z was rounded (slopes change by at most 1.13 for gelu, 0.5 for silu, a step at 0 for relu: there z keeps its sign), dz is rounded
    d8, slope = dy.double().abs(), torch.autograd.functional.jvp(ACTS[act], (z,), (torch.ones_like(z),))[1]
    dz = d8 * slope.abs()
    dz_off = d8 * (1.2 * (half * z.abs() + sum_off + tiny) + 2.0 ** -18) + half * dz + tiny
    if act == "relu":      # z within its error of 0 may come out on the other side
        dz_off = dz_off + d8 * (z.abs() <= sum_off)
    for got, ref, off, k_sum in ((dx, gx, dz_off @ w.double().abs(), n * 2.0 ** -23 * (dz @ w.double().abs())),
                                 (dw, gw, dz_off.T @ x.double().abs(), m * 2.0 ** -23 * (dz.T @ x.double().abs())),
                                 (db, gb, dz_off.sum(0), m * 2.0 ** -23 * dz.sum(0))):
        assert bool(((got.double() - ref).abs() <= half * ref.abs() + 1.01 * (off + k_sum) + tiny).all())


@pytest.mark.parametrize("act", ["gelu", "gelu_tanh", "silu", "relu"])
def test_gradients_agree_with_differences(act):
    m, k, n = 24, 40, 48
    x, w, dy = _normal((m, k), 1, torch.float16), _normal((n, k), 2, torch.float16, k ** -0.5), _normal((m, n), 3, torch.float16)
    b = _normal((n,), 4, torch.float32)
    layer = Linear16(w, b, act)
    layer.forward(x, training=True)
    dx, dw, db = layer.backward(dy, grad_dtype=torch.float32)

    def value(x, w, b):
        return float((ACTS[act](x @ w.T + b) * dy.double()).sum())
    base, h = [t.double() for t in (x, w, b)], 1e-6
    for i, grad in enumerate((dx, dw, db)):
        way = torch.randn(base[i].shape, dtype=torch.float64, device="cuda", generator=_gen(9 + i))
        at = [value(*[t + s * h * way if j == i else t for j, t in enumerate(base)]) for s in (1, -1)]
        want = (at[0] - at[1]) / (2 * h)
        terms = (grad.double() * way).abs().sum()
        assert abs(float((grad.double() * way).sum()) - want) <= float(terms) * 2.0 ** -9      # halves of fp16: z, dz and dx rounded by 2^-11 each


@pytest.mark.parametrize("m,n", [(1, 1000), (12, 1000), (40, 1000), (200, 1000), (200, 1001)])      # the forms of the product
@pytest.mark.parametrize("dtype", HALVES)
def test_gelu_to_a_fraction_of_itself(m, n, dtype):
    """Down the negative tail, too, where gelu is small: z comes as the bias and is exact.  Phi is good to 2^-19 (its fit 2^-22.9, a reciprocal and a power of two a few units of 2^-23, a
    dozen operations of 2^-24), and z^2 / 2 in the exponent is off by two roundings and a constant's, 2^-23 of itself."""
    z = torch.linspace(-12.9, 9.0, n, device="cuda")
    z8 = z.double()
    want = 0.5 * z8 * torch.erfc(-z8 * 0.5 ** 0.5)
    off = want.abs() * (2.0 ** -19 + z8.square() * 2.0 ** -24)
    x, w = torch.zeros(m, 64, dtype=dtype, device="cuda"), torch.zeros(n, 64, dtype=dtype, device="cuda")
    assert bool(((linear16(x, w, z, "gelu", out_dtype=torch.float32).double() - want).abs() <= off).all())
    tiny = 2.0 ** -25 if dtype is torch.float16 else 0.0
    assert bool(((linear16(x, w, z, "gelu").double() - want).abs() <= 1.001 * off + torch.finfo(dtype).eps / 2 * want.abs() + tiny).all())


@pytest.mark.parametrize("dtype", HALVES)
def test_the_slope_of_gelu_to_a_fraction_of_its_terms(dtype):
    """Phi(z) + z phi(z), as the gradient of the bias of a single token in 32 bits; the same errors of either term.  z is kept in 16 bits: whole multiples of 2^-4 are exact."""
    z = torch.arange(-206, 144, device="cuda").float() / 16
    n = z.numel()
    layer = Linear16(torch.zeros(n, 64, dtype=dtype, device="cuda"), z, "gelu")
    layer.forward(torch.zeros(1, 64, dtype=dtype, device="cuda"), training=True)
    _, _, db = layer.backward(torch.ones(1, n, dtype=dtype, device="cuda"), grad_dtype=torch.float32)
    z8 = z.double()
    phi, tail = 0.5 * torch.erfc(-z8 * 0.5 ** 0.5), z8 * torch.exp(-0.5 * z8.square()) * (2 * torch.pi) ** -0.5
    assert bool(((db.double() - (phi + tail)).abs() <= (phi + tail.abs()) * (2.0 ** -19 + z8.square() * 2.0 ** -24)).all())


@pytest.mark.parametrize("act", ["none", "gelu", "silu", "relu", "gelu_tanh"])
@pytest.mark.parametrize("m", [4, 40, 200])
def test_no_inner_entries(act, m):
    """k = 0: the activation of the bias, and the residual."""
    x, w = torch.empty(m, 0, dtype=torch.bfloat16, device="cuda"), torch.empty(70, 0, dtype=torch.bfloat16, device="cuda")
    b, r = _normal((70,), 1, torch.float32), _normal((m, 70), 2, torch.bfloat16)
    got, want = linear16(x, w, b, act, r, out_dtype=torch.float32).double(), ACTS[act](b.double()) + r.double()
    assert bool(((got - want).abs() <= 2.0 ** -19 * (1 + want.abs())).all())
    layer = Linear16(w, b, act)
    layer.forward(x, training=True)
    dx, dw, db = layer.backward(r)
    assert dx.shape == (m, 0) and dw.shape == (70, 0) and db.shape == (70,)


@pytest.mark.parametrize("m,n", [(0, 70), (70, 0)])
def test_nothing(m, n):
    x, w = _whole((m, 32), 1, torch.bfloat16), _whole((n, 32), 2, torch.bfloat16)
    layer = Linear16(w, torch.zeros(n, device="cuda"), "gelu")
    assert linear16(x, w).shape == (m, n) and layer.forward(x, training=True).shape == (m, n)
    dx, dw, db = layer.backward(torch.empty(m, n, dtype=torch.bfloat16, device="cuda"))
    assert dx.shape == (m, 32) and dw.shape == (n, 32) and db.shape == (n,)
    assert not (dx.any() or dw.any() or db.any())


@pytest.mark.parametrize("m", [3, 40, 300])
def test_infinities_and_nans_stay_in_their_rows(m):
    x, w = _whole((m, 72), 1, torch.bfloat16), _whole((200, 72), 2, torch.bfloat16)
    clean = linear16(x, w, out_dtype=torch.float32)
    x[1, 70] = float("nan")
    w[5, 3] = float("inf")
    got = linear16(x, w, out_dtype=torch.float32)
    assert bool(got[1].isnan().all())
    rest = [i for i in range(m) if i != 1]
    cols = [i for i in range(200) if i != 5]
    assert torch.equal(got[rest][:, cols], clean[rest][:, cols]) and not bool(got[rest][:, 5].isfinite().any())


def test_weights_in_32_bits_are_rounded_once():
    w, x, b = _normal((130, 77), 1, torch.float32), _normal((200, 77), 2, torch.float16), _normal((130,), 3, torch.float32)
    assert torch.equal(Linear16(w, b, dtype=torch.float16).forward(x), linear16(x, w.to(torch.float16), b))
    layer = Linear16(w)
    assert torch.equal(layer.weight, w.to(torch.bfloat16))
    layer.set_weight(2 * w)
    assert torch.equal(layer.weight, (2 * w).to(torch.bfloat16))
    assert torch.equal(Linear16(w[:, 5:]).weight, w[:, 5:].to(torch.bfloat16))


def test_same_bits_every_time():
    x, w, dy = _normal((1000, 700), 1, torch.bfloat16), _normal((600, 700), 2, torch.bfloat16), _normal((1000, 600), 3, torch.bfloat16)
    layer = Linear16(w, torch.zeros(600, device="cuda"), "gelu")

    def step():
        return layer.forward(x, training=True), *layer.backward(dy, grad_dtype=torch.float32)
    first = step()
    for _ in range(5):
        assert all(torch.equal(a, b) for a, b in zip(first, step()))


def test_refusals():
    x, w, r = _whole((30, 64), 1, torch.bfloat16), _whole((48, 64), 2, torch.bfloat16), _whole((30, 48), 3, torch.bfloat16)
    with pytest.raises(TypeError):
        linear16(x.float(), w)
    with pytest.raises(TypeError):
        linear16(x, w.half())
    with pytest.raises(ValueError):
        linear16(x, w[:, :60])
    with pytest.raises(ValueError):
        linear16(x, w, activation="tanh")
    with pytest.raises(ValueError):
        linear16(x, w, torch.zeros(47, device="cuda"))
    with pytest.raises(ValueError):
        linear16(x, w, torch.zeros(48, device="cuda", dtype=torch.bfloat16))
    with pytest.raises(ValueError):
        linear16(x, w, residual=r[:29])
    with pytest.raises(TypeError):
        linear16(x, w, residual=r.float())
    with pytest.raises(TypeError):
        linear16(x, w, out_dtype=torch.float16)
    with pytest.raises(ValueError):
        linear16(x, w, out=r[:29])
    with pytest.raises(ValueError):
        linear16(x.cpu(), w)
    with pytest.raises(ValueError):
        linear16(x, w.cpu())
    with pytest.raises(ValueError):
        linear16(x[0], w)
    square = _whole((64, 64), 1, torch.bfloat16)
    for bad in (dict(out=square), dict(residual=square[:30], out=square[1:31])):      # an output over the input, over part of the residual
        with pytest.raises(DsqError):
            linear16(square[:30], square, **bad) if "residual" in bad else linear16(square, square, **bad)
    layer = Linear16(w, activation="relu")
    with pytest.raises(RuntimeError):
        layer.backward(r)
    layer.forward(x)
    with pytest.raises(RuntimeError):
        layer.backward(r)
    layer.forward(x, training=True)
    with pytest.raises(TypeError):
        layer.backward(r.float())
    with pytest.raises(ValueError):
        layer.backward(r[:, :40])
    with pytest.raises(TypeError):
        layer.backward(r, grad_dtype=torch.float16)
    with pytest.raises(ValueError):
        layer.backward(r, dw=torch.empty(48, 63, device="cuda"))
    with pytest.raises(TypeError):
        Linear16(w.float(), dtype=torch.float32)

"""Norms around a residual connection, forward and backward, against arithmetic in 64 bits.

Tolerances: results are rounded by half a step of their type; in 32 bits, a row's sums pass at most 32 additions in a thread, 5 across a warp and 32 across warps and CTAs, 70
roundings of 2^-24 or 2^-17 of the sum of magnitudes, and a dozen operations follow (2^-20).  OFF = 2^-16 covers both; it multiplies the magnitudes of the terms that
make up a value, which the reference works out beside the value.
"""
import pytest
import torch

from paper_1905_05957_b200 import DsqError, ResidualNorm
from tests.test_gpu_dropout import kept

pytestmark = pytest.mark.gpu
OFF = 2.0 ** -16
TYPES = [(torch.float32, torch.float32), (torch.bfloat16, torch.bfloat16), (torch.float16, torch.float16), (torch.bfloat16, torch.float32), (torch.float16, torch.float32)]


def _normal(shape, seed, dtype=torch.float32, scale=1.0, shift=0.0):
    return (shift + scale * torch.randn(shape, device="cuda", generator=torch.Generator(device="cuda").manual_seed(seed))).to(dtype)


def _half(dtype):
    return torch.finfo(dtype).eps / 2


def _tiny(dtype):
    return 2.0 ** -25 if dtype is torch.float16 else 0.0


def _params(cols, norm, post, pre, groups, biases):
    p = {}
    if post:
        p["post_weight"] = _normal((cols,), 11, scale=0.3, shift=1.0)
        if biases:
            p["post_bias"] = _normal((cols,), 12, scale=0.3)
    if groups:
        p["gate"] = _normal((groups, cols), 13)
    if pre:
        p["pre_weight"] = _normal((cols,), 14, scale=0.3, shift=1.0)
        if biases:
            p["pre_bias"] = _normal((cols,), 15, scale=0.3)
    return p


def _norm64(v, w, b, norm, eps):
    """Value and magnitude of terms of a norm of rows."""
    c = v - v.mean(1, keepdim=True) if norm == "layer" else v
    r = (c.square().mean(1, keepdim=True) + eps).rsqrt()
    out = c * r * w
    size = (out.abs() + (v.abs().mean(1, keepdim=True) * r * w.abs() if norm == "layer" else 0)).detach()
    return (out, size) if b is None else (out + b, size + b.detach().abs())


def reference(y, x, leaves, norm, scale, eps, mask, keep_scale, groups):
    """h, n, and for each the magnitude of what is added up in it."""
    u, size = y, y.detach().abs()
    if "post_weight" in leaves:
        u, size = _norm64(y, leaves["post_weight"], leaves.get("post_bias"), norm, eps)
    if groups:
        g = leaves["gate"].reshape(groups, -1).repeat_interleave(y.shape[0] // groups, 0)
        u, size = u * g, size * g.detach().abs()
    if mask is not None:
        u, size = torch.where(mask, u * keep_scale, 0.0), size * mask * keep_scale
    h = u if x is None else scale * x + u
    size = size if x is None else size + (scale * x.detach()).abs()
    n = n_size = None
    if "pre_weight" in leaves:
        n, n_size = _norm64(h, leaves["pre_weight"], leaves.get("pre_bias"), norm, eps)
        hd = h.detach()
        c = hd - hd.mean(1, keepdim=True) if norm == "layer" else hd
        r = (c.square().mean(1, keepdim=True) + eps).rsqrt()
        w = leaves["pre_weight"].detach().abs()
        # an error of h moves its entry, the mean and the size of the row
        n_size = n_size + r * w * (size + size.mean(1, keepdim=True) + (c * r).abs() * (size * (c * r).abs()).mean(1, keepdim=True))
    return h, size, n, n_size


CASES = [  # rows, cols, norm, post, pre, groups, biases, p, x
    (1, 1, "rms", True, True, 0, True, 0.0, True), (1, 4096, "rms", True, True, 0, False, 0.0, True), (5, 7, "layer", True, True, 0, True, 0.3, True),
    (3, 8, "layer", False, True, 3, True, 0.0, True), (16, 33, "rms", True, False, 4, False, 0.5, True), (40, 130, "layer", True, True, 2, False, 0.1, True),
    (37, 768, "layer", False, True, 0, True, 0.1, True), (300, 256, "rms", True, True, 5, False, 0.1, True), (64, 1153, "layer", True, True, 1, True, 0.0, True),
    (20, 2056, "rms", True, True, 20, False, 0.2, True), (33, 4100, "layer", True, True, 3, True, 0.1, True), (9, 8192, "rms", True, True, 0, False, 0.0, True),
    (6, 12296, "layer", True, True, 2, True, 0.1, True), (4, 32768, "rms", True, True, 0, False, 0.0, True), (3, 20001, "layer", True, True, 3, True, 0.0, True),
    (50, 512, "rms", False, True, 0, False, 0.0, False), (50, 520, "layer", False, True, 0, True, 0.0, False), (12, 100, "rms", False, False, 1, False, 0.4, True),
    (700, 64, "layer", True, False, 7, True, 0.0, False), (2000, 96, "rms", True, True, 500, False, 0.1, True), (400, 48, "rms", True, True, 400, False, 0.0, True),
    (15, 40, "rms", False, False, 0, False, 0.25, True),
]


@pytest.mark.parametrize("types", TYPES, ids=str)
@pytest.mark.parametrize("case", CASES, ids=str)
def test_forward_and_backward(case, types):
    rows, cols, norm, post, pre, groups, biases, p, with_x = case
    dtype, stream = types
    if not with_x:
        stream = dtype
    scale, eps, seed, step, layer = 0.75, 1e-5, 77, 5, 2
    y = _normal((rows, cols), 1, dtype, 2.0, 0.5)
    x = _normal((rows, cols), 2, stream, 1.0, -0.25) if with_x else None
    params = _params(cols, norm, post, pre, groups, biases)
    op = ResidualNorm(norm, **params, residual_scale=scale, eps=eps, p=p, seed=seed, layer=layer)
    leaves = {k: v.double().requires_grad_() for k, v in params.items()}
    y8, x8 = y.double().requires_grad_(), None if x is None else x.double().requires_grad_()
    mask = kept(rows, cols, p, seed, step, layer) if p else None
    keep_scale = 65536 / (65536 - round(p * 65536))
    h8, h_size, n8, n_size = reference(y8, x8, leaves, norm, scale, eps, mask, keep_scale, groups)
    for training in (False, True):
        h, n = op.forward(y, x, step=step, training=training)
        assert h.dtype is stream and bool(((h.double() - h8).abs() <= _half(stream) * h8.abs() + OFF * h_size + _tiny(stream)).all())
        assert (n is None) == (not pre)
        if pre:
            assert n.dtype is dtype and bool(((n.double() - n8).abs() <= _half(dtype) * n8.abs() + OFF * n_size + _tiny(dtype)).all())
    dh = _normal((rows, cols), 3, stream)
    dn = _normal((rows, cols), 4, dtype) if pre else None
    for given in [(dh, dn)] + ([(None, dn)] if pre else []):
        ends = [(e, g.double()) for e, g in zip((h8, n8), given) if g is not None]
        inputs = [y8] + ([x8] if with_x else []) + list(leaves.values())
        want = torch.autograd.grad([e for e, _ in ends], inputs, [g for _, g in ends], retain_graph=True, allow_unused=True)
        want = dict(zip(["y"] + (["x"] if with_x else []) + list(leaves), want))
        dy, dx, grads = op.backward(*given)
        assert dy.dtype is dtype and set(grads) == set(leaves) and (dx is None) == (not with_x)
        # an error against the row's or the column's largest value: the terms of a row's gradient are of its size, short rows may cancel (down to nothing where a
        # layer norm has one column), so what the norms divide by and multiply with counts
        for got, ref, half, tiny in [(dy, want["y"], _half(dtype), _tiny(dtype))] + ([(dx, want["x"], _half(stream), _tiny(stream))] if with_x else []):
            size = _back_size(y8.detach(), None if x is None else x8.detach(), {k: v.detach() for k, v in leaves.items()}, given, norm, scale, eps, mask, keep_scale, groups,
                              "y" if got is dy else "x")
            assert bool(((got.double() - ref).abs() <= half * ref.abs() + OFF * size + tiny).all())
        for name, got in grads.items():
            ref = want[name] if want[name] is not None else torch.zeros_like(leaves[name])
            assert got.shape == params[name].shape
            size = _column_size(y8.detach(), None if x is None else x8.detach(), {k: v.detach() for k, v in leaves.items()}, given, norm, scale, eps, mask, keep_scale, groups,
                                name)
            assert bool(((got.double() - ref).abs() <= OFF * size).all()), name


def _hat(v, norm, eps):
    c = v - v.mean(1, keepdim=True) if norm == "layer" else v
    r = (c.square().mean(1, keepdim=True) + eps).rsqrt()
    return c * r, r, v.abs().mean(1, keepdim=True) * r if norm == "layer" else 0.0


def _pull(t, hat, r, norm):
    """Magnitude of what is added up in r (t - mean(t) - hat mean(t hat)); t: magnitudes."""
    return r * (t + t.mean(1, keepdim=True) + hat.abs() * (t * hat.abs()).mean(1, keepdim=True))


def _sizes(y, x, leaves, given, norm, scale, eps, mask, keep_scale, groups):
    """Magnitudes along the backward pass: of d (the gradient of h), of the normalised rows with what their errors add, and so on."""
    one = torch.ones_like(y)
    hat1, r1, m1 = _hat(y, norm, eps) if "post_weight" in leaves else (y, one[:, :1], 0.0)
    v = hat1.abs() + m1
    if "post_weight" in leaves:
        v = v * leaves["post_weight"].abs() + (leaves["post_bias"].abs() if "post_bias" in leaves else 0.0)
    g = leaves["gate"].reshape(groups, -1).repeat_interleave(y.shape[0] // groups, 0).abs() if groups else one
    k = mask * keep_scale if mask is not None else one
    dh, dn = given
    d = dh.double().abs() if dh is not None else torch.zeros_like(y)
    hat2_size = None
    if dn is not None:
        h, h_size, _, _ = reference(y, x, leaves, norm, scale, eps, mask, keep_scale, groups)
        hat2, r2, m2 = _hat(h, norm, eps)
        # the normalised row and how far an error of OFF in the terms of h moves it
        hat2_size = hat2.abs() + m2 + r2 * (h_size + h_size.mean(1, keepdim=True)) + hat2.abs() * (h_size * hat2.abs()).mean(1, keepdim=True) * r2
        t = dn.double().abs() * leaves["pre_weight"].abs()
        d = d + _pull(t, hat2_size, r2, norm) * (1 + (h_size * hat2.abs()).mean(1, keepdim=True) * r2)
    return hat1.abs() + m1, r1, v, g, k, d, hat2_size


def _back_size(y, x, leaves, given, norm, scale, eps, mask, keep_scale, groups, which):
    hat1, r1, v, g, k, d, _ = _sizes(y, x, leaves, given, norm, scale, eps, mask, keep_scale, groups)
    if which == "x":
        return abs(scale) * d
    d = d * k * g
    return _pull(d * leaves["post_weight"].abs(), hat1, r1, norm) if "post_weight" in leaves else d


def _column_size(y, x, leaves, given, norm, scale, eps, mask, keep_scale, groups, name):
    hat1, r1, v, g, k, d, hat2 = _sizes(y, x, leaves, given, norm, scale, eps, mask, keep_scale, groups)
    if name == "gate":
        return (d * k * v).reshape(groups, -1, y.shape[1]).sum(1)
    if name == "post_weight":
        return (d * k * g * hat1).sum(0)
    if name == "post_bias":
        return (d * k * g).sum(0)
    dn = given[1].double().abs() if given[1] is not None else torch.zeros_like(y)
    return (dn * hat2).sum(0) if name == "pre_weight" else dn.sum(0)


@pytest.mark.parametrize("norm", ["rms", "layer"])
def test_gradients_agree_with_differences(norm):
    rows, cols, groups = 6, 40, 2
    params = _params(cols, norm, True, True, groups, True)
    y, x, dh, dn = (_normal((rows, cols), s) for s in (1, 2, 3, 4))
    op = ResidualNorm(norm, **params, residual_scale=0.8, p=0.25, seed=3)
    op.forward(y, x, training=True)
    dy, dx, grads = op.backward(dh, dn)
    mask = kept(rows, cols, 0.25, 3, 0, 0)
    names = list(params)
    base = [y.double(), x.double()] + [params[k].double() for k in names]

    def value(at):
        h, _, n, _ = reference(at[0], at[1], dict(zip(names, at[2:])), norm, 0.8, 1e-5, mask, 65536 / 49152, groups)
        return float((h * dh.double()).sum() + (n * dn.double()).sum())
    for i, grad in enumerate([dy, dx] + [grads[k] for k in names]):
        way = torch.randn(base[i].shape, dtype=torch.float64, device="cuda", generator=torch.Generator(device="cuda").manual_seed(20 + i))
        e = 1e-6
        at = [value([t + s * e * way if j == i else t for j, t in enumerate(base)]) for s in (1, -1)]
        terms = float((grad.double() * way).abs().sum())
        assert abs(float((grad.double() * way).sum()) - (at[0] - at[1]) / (2 * e)) <= 2.0 ** -14 * terms


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("pad,offset", [(8, 0), (3, 1), (16, 4), (0, 5)])
def test_rows_within_wider_rows(pad, offset, dtype):
    rows, cols = 23, 100
    params = _params(cols, "layer", True, True, 1, True)

    def within(t):
        buf = torch.full((offset + rows * (cols + pad) + 32,), 3.0, dtype=dtype, device="cuda")
        v = buf.as_strided((rows, cols), (cols + pad, 1), offset)
        v.copy_(t)
        return v, buf
    tight = [_normal((rows, cols), s, dtype) for s in (1, 2, 3, 4)]
    op, other = (ResidualNorm("layer", **params, p=0.1, seed=1) for _ in range(2))
    want = op.forward(tight[0], tight[1], training=True)
    back = op.backward(tight[2], tight[3])
    wide = [within(t)[0] for t in tight]
    (h, hb), (n, nb) = within(tight[0]), within(tight[0])
    other.forward(wide[0], wide[1], training=True, h=h, n=n)
    got = other.backward(wide[2], wide[3])
    assert torch.equal(h, want[0]) and torch.equal(n, want[1])
    assert torch.equal(got[0], back[0]) and torch.equal(got[1], back[1]) and all(torch.equal(got[2][k], back[2][k]) for k in params)
    for v, buf in ((h, hb), (n, nb)):
        v.fill_(3.0)
        assert bool((buf == 3.0).all())


def test_parameters_on_no_boundary():
    """Vectors that begin four bytes behind a 16-byte boundary, as slices of a flat model do."""
    rows, cols = 30, 256
    params = _params(cols, "layer", True, True, 3, True)
    odd = {}
    for k, v in params.items():
        buf = torch.empty(v.numel() + 1, device="cuda")
        buf[1:].copy_(v.reshape(-1))
        odd[k] = buf[1:].view(v.shape)
    y, x, dh, dn = (_normal((rows, cols), s, torch.bfloat16) for s in (1, 2, 3, 4))
    got = []
    for p in (params, odd):
        op = ResidualNorm("layer", **p)
        got.append((*op.forward(y, x, training=True), *op.backward(dh, dn)))
    assert all(torch.equal(a, b) for a, b in zip(got[0][:4], got[1][:4])) and all(torch.equal(got[0][4][k], got[1][4][k]) for k in params)


def test_given_outputs_and_in_place():
    rows, cols = 64, 512
    params = _params(cols, "rms", True, True, 0, False)
    op = ResidualNorm("rms", **params)
    y, x, dh, dn = (_normal((rows, cols), s, torch.bfloat16) for s in (1, 2, 3, 4))
    h, n = op.forward(y, x, training=True)
    row = torch.zeros(5 * cols, device="cuda")
    dy, dx, grads = op.backward(dh, dn, out={"pre_weight": row[cols:2 * cols], "post_weight": row[3 * cols:4 * cols]})
    _, _, again = op.backward(dh, dn)
    assert all(torch.equal(grads[k], again[k]) for k in params) and torch.equal(row[cols:2 * cols], again["pre_weight"])
    assert not row[:cols].any() and not row[2 * cols:3 * cols].any() and not row[4 * cols:].any()
    assert op.backward(dh, dn, need_dx=False)[1] is None
    only = op.forward(y, x, need_h=False)
    assert only[0] is None and torch.equal(only[1], n)
    xs, ys = x.clone(), y.clone()
    op.forward(ys, xs, h=xs, n=ys)
    assert torch.equal(xs, h) and torch.equal(ys, n)
    with pytest.raises(ValueError):
        op.forward(y, x, training=True, h=x)


def test_rows_do_not_touch_one_another():
    """An inf or a NaN makes its own row NaN, and nothing else."""
    rows, cols = 40, 300
    op = ResidualNorm("layer", **_params(cols, "layer", True, True, 0, True))
    y, x, dh, dn = (_normal((rows, cols), s) for s in (1, 2, 3, 4))
    clean = [*op.forward(y, x, training=True), *op.backward(dh, dn)[:2]]
    y[7, 100], x[9, 299], dn[11, 0] = float("nan"), float("inf"), float("nan")
    got = [*op.forward(y, x, training=True), *op.backward(dh, dn)[:2]]
    rest = [r for r in range(rows) if r not in (7, 9, 11)]
    assert all(torch.equal(a[rest], b[rest]) for a, b in zip(got, clean))
    assert bool(got[1][7].isnan().all()) and bool(got[1][9].isnan().all()) and bool(got[2][11].isnan().all())


def _formula(y, x, params, norm, eps=1e-5):
    """h and n by the formulas in 32 bits, with what they make of infs and NaNs."""
    def normed(v, which):
        c = v - v.mean(1, keepdim=True) if norm == "layer" else v
        return c * (c.square().mean(1, keepdim=True) + eps).rsqrt() * params[which + "_weight"] + params.get(which + "_bias", 0.0)
    h = x + (normed(y, "post") if "post_weight" in params else y) * params["gate"]
    return h, normed(h, "pre") if "pre_weight" in params else None


@pytest.mark.parametrize("biases", [False, True])
@pytest.mark.parametrize("post,pre", [(True, True), (True, False), (False, True), (False, False)])
@pytest.mark.parametrize("norm", ["rms", "layer"])
def test_what_infs_nans_and_large_rows_become(norm, post, pre, biases):
    """Each follows the formulas, in its row, and in the parameters' gradients in the columns of which a term is one; other rows are as they were."""
    rows, cols = 24, 300
    params = _params(cols, norm, post, pre, 1, biases)
    y, x, dh = (_normal((rows, cols), s) for s in (1, 2, 3))
    dn = _normal((rows, cols), 4) if pre else None
    op = ResidualNorm(norm, **params)
    clean = [t for t in (*op.forward(y, x, training=True), *op.backward(dh, dn)[:2]) if t is not None]
    y[3, 100], y[5, 7], x[8, 299], x[10, 0] = float("nan"), float("inf"), float("-inf"), float("nan")
    y[12], x[13] = 1e19 * torch.sign(y[12]) * (1 + y[12].abs()), 1e19 * torch.sign(x[13]) * (1 + x[13].abs())      # squares sum to 3e40 and more
    touched = [3, 5, 8, 10, 12, 13]
    h, n = op.forward(y, x, training=True)
    for got, want in zip((h, n), _formula(y, x, params, norm)):
        if got is None:
            continue
        assert torch.equal(got.isnan(), want.isnan()) and torch.equal(got.isinf(), want.isinf())
        ok = want.isfinite()
        assert bool(((got - want).abs()[ok] <= 2.0 ** -14 * (1 + want.abs()[ok])).all())
    dy, dx, grads = op.backward(dh, dn)
    rest = [r for r in range(rows) if r not in touched]
    assert all(torch.equal(a[rest], b[rest]) for a, b in zip([t for t in (h, n, dy, dx) if t is not None], clean))
    if post:
        assert bool(dy[3].isnan().all()) and bool(dy[5].isnan().all()) and bool(h[12].isfinite().all())
        assert bool(grads["post_weight"].isnan().all())
        if norm == "rms":      # the finite entries of a row with an inf are 0
            assert bool(h[5, :7].eq(x[5, :7]).all()) != biases
    if not post and not pre:
        assert int(h.isnan().sum()) == 2 and int(h.isinf().sum()) == 2 and bool(dy.isfinite().all()) and int((~grads["gate"].isfinite()).sum()) == 2


def test_gradients_of_an_rms_norm_with_an_inf():
    """The finite entries of its row are 0 and add 0: one column alone is NaN."""
    w = torch.ones(300, device="cuda")
    y, dh = _normal((24, 300), 1), _normal((24, 300), 2)
    y[5, 7] = float("inf")
    op = ResidualNorm("rms", post_weight=w)
    op.forward(y, training=True)
    assert op.backward(dh)[2]["post_weight"].isnan().nonzero().flatten().tolist() == [7]
    op = ResidualNorm("rms", pre_weight=w)
    op.forward(y, training=True)
    assert op.backward(dn=dh)[2]["pre_weight"].isnan().nonzero().flatten().tolist() == [7]


def test_rows_of_zeros_and_large_means():
    op = ResidualNorm("layer", post_weight=torch.ones(512, device="cuda"), eps=1e-5)
    y = torch.zeros(4, 512, device="cuda")
    assert not op.forward(y)[0].any()
    assert not op.forward(y + 1000)[0].any()              # a constant row is its mean
    v = _normal((4, 512), 1, shift=1000.0)
    want = torch.nn.functional.layer_norm(v.double(), (512,), eps=1e-5)
    # entries and their mean are off by half a step of 1000 (2^-15), and so is a row's scale
    assert float((op.forward(v)[0].double() - want).abs().max()) < 2.0 ** -12
    rms = ResidualNorm("rms", pre_weight=torch.ones(512, device="cuda"), eps=1e-6)
    rms.forward(y, training=True)
    dy, _, g = rms.backward(dn=torch.ones(4, 512, device="cuda"))
    assert float((dy - 1000).abs().max()) < 1e-2 and not g["pre_weight"].any()      # 1 / sqrt(eps)


@pytest.mark.parametrize("biases", [False, True])
@pytest.mark.parametrize("post,pre", [(True, False), (False, True), (False, False)])
def test_statistics_of_norms_that_are_not_there(post, pre, biases):
    """Memory that the forward pass leaves as it was has no part in the gradients."""
    rows, cols = 37, 200
    for norm in ("rms", "layer"):
        params = _params(cols, norm, post, pre, 1, biases)
        op = ResidualNorm(norm, **params)
        y, x, dh, dn = (_normal((rows, cols), s) for s in (1, 2, 3, 4))
        got = []
        for poison in (0.0, float("nan"), float("inf")):
            junk = [torch.full((rows, 4), poison, device="cuda") for _ in range(64)]      # what is given back next is one of these
            del junk
            op.forward(y, x, training=True)
            for given in ((dh, dn) if pre else (dh,), (dh,)):
                dy, dx, g = op.backward(*given)
                got.append([dy, dx, *g.values()])
        for i in range(2):
            assert all(bool(t.isfinite().all()) for t in got[i])
            assert all(torch.equal(a, b) for other in got[i + 2::2] for a, b in zip(got[i], other))


@pytest.mark.parametrize("rows,cols", [(5, 8), (33, 200), (7, 333), (3, 4100)])
def test_columns_of_one_buffer(rows, cols):
    """Inputs and outputs side by side in wider rows; what does share memory is refused."""
    buf = torch.zeros(rows, 4 * cols, device="cuda")
    y, x, h, n = (buf[:, i * cols:(i + 1) * cols] for i in range(4))
    y.copy_(_normal((rows, cols), 1))
    x.copy_(_normal((rows, cols), 2))
    op = ResidualNorm("layer", **_params(cols, "layer", True, True, 1, True))
    want = op.forward(y.clone(), x.clone())
    op.forward(y, x, h=h, n=n)
    assert torch.equal(h, want[0]) and torch.equal(n, want[1])
    with pytest.raises(DsqError):
        op.forward(y, x, h=h, n=buf[:, 3 * cols - 1:4 * cols - 1])


def test_no_rows():
    params = _params(64, "rms", True, True, 2, False)
    op = ResidualNorm("rms", **params)
    e = torch.empty(0, 64, device="cuda")
    h, n = op.forward(e, e, training=True)
    dy, dx, grads = op.backward(h, n)
    assert h.shape == n.shape == dy.shape == dx.shape == (0, 64) and not any(g.any() for g in grads.values())


def test_same_bits_every_time():
    params = _params(768, "layer", True, True, 4, True)
    op = ResidualNorm("layer", **params, p=0.1, seed=1)
    y, x, dh, dn = (_normal((4096, 768), s, torch.bfloat16) for s in (1, 2, 3, 4))

    def step():
        a = op.forward(y, x, training=True)
        dy, dx, g = op.backward(dh, dn)
        return [*a, dy, dx, *g.values()]
    first = step()
    for _ in range(5):
        assert all(torch.equal(a, b) for a, b in zip(first, step()))


def test_refusals():
    w, x = torch.ones(64, device="cuda"), _normal((10, 64), 1)
    for bad in (dict(norm="batch"), dict(post_bias=w), dict(pre_bias=w), dict(eps=-1.0), dict(eps=float("nan")), dict(p=1.0), dict(post_weight=w, pre_weight=w[:60]),
                dict(post_weight=w.bfloat16()), dict(post_weight=w.cpu()), dict(gate=torch.ones(2, 2, 64, device="cuda")), dict(pre_weight=w, layer=-1)):
        with pytest.raises(ValueError):
            ResidualNorm(**bad)
    op = ResidualNorm(post_weight=w, gate=torch.ones(3, 64, device="cuda"))
    with pytest.raises(ValueError):
        op.forward(x)                                   # 10 rows are not three runs
    op = ResidualNorm(post_weight=w)
    for bad in (dict(y=x[:, :60]), dict(y=x, x=x[:9]), dict(y=x, n=x.clone()), dict(y=x, need_h=False), dict(y=x, step=-1), dict(y=x[0]), dict(y=x.cpu())):
        with pytest.raises(ValueError):
            op.forward(**bad)
    with pytest.raises(TypeError):
        op.forward(x.double())
    with pytest.raises(TypeError):
        op.forward(x, x.bfloat16())
    with pytest.raises(RuntimeError):
        op.backward(x)
    op.forward(x, training=True)
    for bad in (dict(), dict(dn=x), dict(dh=x[:9]), dict(dh=x, out={"gate": w}), dict(dh=x, out={"post_weight": w[:60]})):
        with pytest.raises(ValueError):
            op.backward(**bad)
    with pytest.raises(TypeError):
        op.backward(x.bfloat16())
    with pytest.raises(ValueError):
        ResidualNorm("rms").forward(torch.zeros(1, 32769, device="cuda"))
    buf = _normal((11, 64), 2)
    with pytest.raises(DsqError):
        op.forward(buf[:10], h=buf[1:])                 # over its input, a row off

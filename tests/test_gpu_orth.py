"""The orthogonalised update on the GPU against its definition in 64 bits.

Tolerance.  The products run on numbers of 11 bits (unit u = 2^-11); the diagonals and the term aX do not.  In the Frobenius
norm a rounded operand of a step changes the step's result by at most about u / 2 of its off-diagonal part, random in sign.
With three such operands a step and later steps passing an error on at no more than its relative size, five steps give
sqrt(15) u / 2 = 1e-3 as their sum of squares; twice that is allowed for what passes on larger (singular values near the
polynomial's steepest places): 2e-3, and the result's own rounding (2^-9 for bfloat16)."""
import pytest
import torch

from paper_1905_05957_b200 import DsqError, OrthUpdate, binding

pytestmark = pytest.mark.gpu
COEF = (3.4445, -4.7750, 2.0315)
TOL = 2e-3
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _exact(u: torch.Tensor, steps=5, eps=1e-7, coef=COEF):
    x = u.double()
    tall = x.shape[-2] > x.shape[-1]
    x = x.mT if tall else x
    x = x / (x.square().sum((-2, -1), keepdim=True).sqrt() + eps)
    for _ in range(steps):
        a = x @ x.mT
        x = coef[0] * x + (coef[1] * a + coef[2] * a @ a) @ x
    return x.mT if tall else x


def _off(got, want):
    return float((got.double() - want).norm() / want.norm())


def _matrix(batch, m, n, kind, seed):
    g = _gen(seed)
    if kind == "noise":
        return torch.randn(batch, m, n, device="cuda", generator=g)
    r = max(1, min(m, n) // 8)
    low = torch.randn(batch, m, r, device="cuda", generator=g) @ torch.randn(batch, r, n, device="cuda", generator=g)
    return low / r ** 0.5 + 0.1 * torch.randn(batch, m, n, device="cuda", generator=g)


SIZES = [(1, 1), (1, 40), (7, 3), (16, 16), (31, 33), (64, 64), (64, 576), (65, 200), (127, 129), (128, 128), (130, 130), (200, 65), (192, 500),
         (256, 1100), (257, 255), (384, 384), (520, 136), (700, 1000), (1000, 512)]


@pytest.mark.parametrize("m,n", SIZES)
@pytest.mark.parametrize("kind", ["noise", "low"])
def test_update_against_64_bits(m, n, kind):
    g = _matrix(1, m, n, kind, m * 1000 + n) * 3e-3
    plan = OrthUpdate(m, n)
    plan.workspace.fill_(0xFF)
    got = plan.update(g, out_dtype=F32)[0]
    assert _off(got, _exact(g[0])) < TOL
    assert torch.equal(plan.update(g, out_dtype=BF16)[0], got.to(BF16))
    assert torch.equal(plan.update(g, out_dtype=F32)[0], got)          # and the same again
    assert not plan.timed_out()


@pytest.mark.parametrize("batch,m,n", [(12, 706, 1202), (1, 1344, 3964), (3, 947, 3707), (2, 2090, 1368), (1, 1250, 1250), (1, 2500, 2500), (6, 512, 512)])
def test_larger_updates_in_every_form_of_product(batch, m, n):
    """Sizes at which the three products of a step are taken in different forms (single CTAs, pairs, split), which say how much of
    the symmetric matrices between them is written."""
    g = _matrix(batch, m, n, "low", m)
    plan = OrthUpdate(m, n, batch=batch)
    plan.workspace.fill_(0xFF)                 # NaN in 16 bits: nothing that was not written may be read
    got = plan.update(g, out_dtype=F32)
    for i in range(batch):
        assert _off(got[i], _exact(g[i])) < TOL
    assert torch.equal(plan.update(g, out_dtype=F32), got) and not plan.timed_out()


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("nesterov", [True, False])
@pytest.mark.parametrize("m,n", [(96, 160), (77, 45), (130, 261)])
def test_momentum_and_direction(dtype, nesterov, m, n):
    mu = 0.9
    plan = OrthUpdate(m, n, batch=2, momentum=mu, nesterov=nesterov)
    buf = _matrix(2, m, n, "low", 3)
    want_buf = buf.clone()
    for t in range(3):
        g = _matrix(2, m, n, "noise", 10 + t).to(dtype)
        got = plan.update(g, buf, out_dtype=F32)
        want_buf = want_buf * mu + g.float()                 # two roundings, as documented: bit for bit
        assert torch.equal(buf, want_buf)
        u = g.float() + mu * want_buf if nesterov else want_buf
        for i in range(2):
            assert _off(got[i], _exact(u[i])) < TOL


@pytest.mark.parametrize("batch,m,n", [(4, 64, 576), (12, 100, 100), (3, 300, 140), (70, 24, 30)])
def test_batches_equal_single_matrices(batch, m, n):
    g = _matrix(batch, m, n, "low", batch) * (10.0 ** torch.linspace(-6, 3, batch, device="cuda"))[:, None, None]
    got = OrthUpdate(m, n, batch=batch).update(g, out_dtype=F32)
    one = OrthUpdate(m, n)
    for i in range(batch):
        assert torch.equal(got[i], one.update(g[i].contiguous(), out_dtype=F32)[0])
        assert _off(got[i], _exact(g[i])) < TOL


@pytest.mark.parametrize("batch,m,n", [(1, 64, 2048), (2000, 7, 3), (3000, 1, 40), (300, 64, 576), (900, 33, 31), (160, 2048, 20)])
def test_small_matrices_are_as_exact_in_any_batch(batch, m, n):
    """Products of 22 bits: three operands a step, five steps, each off by 2^-22 at most, passed on by up to a = 3.4 a step in the
    worst direction.  Documented: 1e-5."""
    g = _matrix(batch, m, n, "low", batch)
    got = OrthUpdate(m, n, batch=batch).update(g, out_dtype=F32)
    want = _exact(g)
    off = (got.double() - want).flatten(1).norm(dim=1) / want.flatten(1).norm(dim=1)
    assert float(off.max()) < 1e-5


@pytest.mark.parametrize("m,n", [(50, 90), (90, 50), (128, 256)])
@pytest.mark.parametrize("lead", [0, 1, 4])
def test_slices_of_a_flat_vector_and_the_model_update(m, n, lead):
    """Three matrices at one distance inside flat g, momentum and x vectors, as the step lays its model out; what lies between
    them is not touched."""
    batch, gap = 3, 13 if lead else 16
    stride, gamma, decay = m * n + gap, 0.02, 0.1
    d = lead + batch * stride
    gen = _gen(m + lead)
    g, buf, x = (torch.randn(d, device="cuda", generator=gen) for _ in range(3))
    buf0, x0 = buf.clone(), x.clone()
    plan = OrthUpdate(m, n, batch=batch, stride=stride)
    out = plan.update(g[lead:], buf[lead:], out_dtype=F32, x=x[lead:], gamma=gamma, decay=decay)
    inside = torch.zeros(d, dtype=torch.bool, device="cuda")
    for i in range(batch):
        inside[lead + i * stride: lead + i * stride + m * n] = True
    assert torch.equal(buf[~inside], buf0[~inside]) and torch.equal(x[~inside], x0[~inside])
    mats = lambda v: torch.stack([v[lead + i * stride: lead + i * stride + m * n].view(m, n) for i in range(batch)])  # noqa: E731
    want_buf = mats(buf0) * 0.95 + mats(g)
    assert torch.equal(mats(buf), want_buf)
    u = mats(g) + 0.95 * want_buf
    scale = max(1.0, m / n) ** 0.5
    for i in range(batch):
        assert _off(out[i], _exact(u[i])) < TOL
    # x from the returned update: the rate and the factor 1 - gamma decay as 32-bit numbers, one rounding an operation
    want_x = mats(x0).double() * (1 - gamma * decay) - gamma * scale * out.double()
    assert ((mats(x).double() - want_x).abs() <= 4 * 2.0 ** -24 * (mats(x0).double().abs() + want_x.abs() + 1)).all()
    x2 = x0.clone()
    assert plan.update(g[lead:], buf0[lead:], out_dtype=None, x=x2[lead:], gamma=gamma, decay=decay) is None
    assert torch.equal(x2, x)


@pytest.mark.parametrize("sigma", [1e-30, 1e-6, 1.0, 1e10, 1e25])
def test_scale_of_the_gradient_does_not_matter(sigma):
    g = _matrix(1, 80, 120, "low", 1)
    got = OrthUpdate(80, 120, eps=0.0).update(g * sigma, out_dtype=F32)[0]
    assert _off(got, _exact(g[0] * sigma, eps=0.0)) < TOL


def test_zero_one_entry_and_not_finite():
    plan = OrthUpdate(40, 72, batch=4)
    g = torch.zeros(4, 40, 72, device="cuda")
    g[1, 3, 5] = -2.0
    g[2] = _matrix(1, 40, 72, "noise", 2)[0]
    g[3] = g[2]
    g[3, 1, 1] = float("nan")
    got = plan.update(g, out_dtype=F32)
    assert (got[0] == 0).all()
    assert _off(got[1], _exact(g[1])) < TOL and int((got[1] != 0).sum()) == 1
    assert _off(got[2], _exact(g[2])) < TOL            # its neighbour's NaN stays there
    assert torch.isnan(got[3]).any()
    g[3, 1, 1] = float("inf")
    assert not torch.isfinite(plan.update(g, out_dtype=F32)[3]).all()


@pytest.mark.parametrize("steps", [1, 2, 3, 8])
def test_other_steps_and_coefficients(steps):
    coef = (1.5, -0.5, 0.0)                      # the cubic iteration, which converges to singular values of one
    g = _matrix(1, 60, 90, "noise", 4)
    got = OrthUpdate(60, 90, steps=steps, coef=coef).update(g, out_dtype=F32)[0]
    assert _off(got, _exact(g[0], steps=steps, coef=coef)) < TOL
    got = OrthUpdate(90, 60, steps=steps).update(g.mT.contiguous(), out_dtype=F32)[0]
    assert _off(got, _exact(g[0].T, steps=steps)) < TOL * max(1, steps / 5)


def test_the_result_is_nearly_orthogonal():
    g = _matrix(1, 96, 400, "noise", 8)
    s = torch.linalg.svdvals(OrthUpdate(96, 400).update(g, out_dtype=F32)[0].double())
    assert 0.6 < float(s.min()) and float(s.max()) < 1.3


def test_another_stream():
    g = _matrix(1, 300, 500, "low", 8)
    plan = OrthUpdate(300, 500)
    want = plan.update(g, out_dtype=F32)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        got = [plan.update(g, out_dtype=F32) for _ in range(10)]
    s.synchronize()
    assert all(torch.equal(v, want) for v in got)


@pytest.mark.parametrize("m,n", [(48, 100), (256, 320)])
def test_in_a_captured_graph(m, n):
    g, buf = _matrix(1, m, n, "low", 1), torch.zeros(1, m, n, device="cuda")
    plan, out = OrthUpdate(m, n), torch.empty(1, m, n, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        plan.update(g, buf, out=out)
    want_buf = torch.zeros_like(buf)
    other = OrthUpdate(m, n)
    for t in range(3):
        g.copy_(_matrix(1, m, n, "low", 5 + t))
        graph.replay()
        want = other.update(g, want_buf, out_dtype=F32)
        torch.cuda.synchronize()
        assert torch.equal(out, want) and torch.equal(buf, want_buf)


def test_refusals():
    for kw in (dict(rows=0, cols=4), dict(rows=4, cols=0), dict(rows=4, cols=4, batch=0), dict(rows=4, cols=4, steps=0),
               dict(rows=4, cols=4, steps=33), dict(rows=4, cols=4, momentum=float("nan")), dict(rows=4, cols=4, eps=-1.0),
               dict(rows=4, cols=4, stride=15), dict(rows=(1 << 20) + 1, cols=1)):
        with pytest.raises(DsqError) as e:
            OrthUpdate(**kw)
        assert e.value.code == binding.DS_ERR_INVALID_ARG
    plan = OrthUpdate(8, 16)
    g = torch.randn(8, 16, device="cuda")
    with pytest.raises(ValueError):
        plan.update(g[:7])
    with pytest.raises(ValueError):
        plan.update(g.T)
    with pytest.raises(ValueError):
        plan.update(g.double())
    with pytest.raises(ValueError):
        plan.update(g, momentum=g.to(BF16))
    with pytest.raises(ValueError):
        plan.update(g, out=torch.empty(8, 16, dtype=F16, device="cuda"))
    with pytest.raises(DsqError):
        plan.update(g, out_dtype=None)                    # nothing to write
    with pytest.raises(DsqError):
        plan.update(g, x=g.clone(), gamma=float("inf"))
    lib, p = binding.load_library(), g.data_ptr()
    assert lib.ds_orth_update(plan.handle, p + 2, 0, None, p, 0, None, 0.0, 0.0, None) == binding.DS_ERR_ALIGN
    assert lib.ds_orth_update(plan.handle, p, 9, None, p, 0, None, 0.0, 0.0, None) == binding.DS_ERR_INVALID_ARG
    assert lib.ds_orth_update(None, p, 0, None, p, 0, None, 0.0, 0.0, None) == binding.DS_ERR_INVALID_ARG
    assert lib.ds_orth_destroy(None) == binding.DS_ERR_INVALID_ARG
    torch.cuda.synchronize()

"""The orthogonalised update of matrices that are far from full rank, against its definition in 64 bits: gradients of dead units, of
embeddings, of few samples.  Their null space is where an update goes wrong: the step multiplies what roundings leave there by
a = 3.44, four times over.

Tolerance of the general form.  What is left there by the two last steps' low halves is 2^-12 (1 + a) of the update.  In the other
directions the off-diagonal parts of A and B are rounded to 11 bits; entries that are all alike (few rows, equal ones) are rounded alike,
by 2^-12 at most, so a step is off by 2^-12 (|b s^2 + c s^4| + |b s^2 + 2 c s^4|) <= 2^-12 (2.8 + 1.4), X's own rounding in A adds
about as much as the latter, and the result of a step is at least 0.7: 2e-3 a step, 1e-2 after five.

Tolerance of the form for small matrices (22 bits): 2^-22 of the update multiplied by a four times, from three operands:
sqrt(3) 140 / 2^22 = 6e-5 from the first step and a quarter as much from each later one; 2e-4 is allowed, twice their sum."""
import pytest
import torch

from paper_1905_05957_b200 import OrthUpdate

pytestmark = pytest.mark.gpu
COEF = (3.4445, -4.7750, 2.0315)
TOL, TOL_SMALL = 1e-2, 2e-4
F32 = torch.float32


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _exact(u, steps=5, coef=COEF, eps=1e-7):
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


def _few_rows(m, n, live, rank, noise, seed):
    """`live` rows of the given rank, with noise beside it; the others zero."""
    g = _gen(seed)
    u = torch.zeros(m, n, device="cuda")
    rows = torch.randperm(m, device="cuda", generator=g)[:live]
    low = torch.randn(live, rank, device="cuda", generator=g) @ torch.randn(rank, n, device="cuda", generator=g)
    u[rows] = low / rank ** 0.5 + noise * torch.randn(live, n, device="cuda", generator=g)
    return u


def _one_sample(m, n, seed):
    """The gradient of a softmax layer from one sample: an outer product."""
    g = _gen(seed)
    p = torch.softmax(2 * torch.randn(m, device="cuda", generator=g), 0)
    p[m // 3] -= 1
    return p[:, None] * torch.relu(torch.randn(n, device="cuda", generator=g))[None]


def _check(u, tol, batch=1):
    plan = OrthUpdate(u.shape[-2], u.shape[-1], batch=batch)
    plan.workspace.fill_(0xFF)
    got = plan.update(u, out_dtype=F32)
    want = _exact(u.reshape(batch, *u.shape[-2:]))
    for i in range(batch):
        assert _off(got[i], want[i]) < tol
    assert not plan.timed_out()


@pytest.mark.parametrize("m,n,live,rank,noise", [
    (128, 300, 2, 1, 0.01), (128, 300, 3, 1, 0.003), (128, 512, 8, 1, 0.01), (128, 512, 8, 1, 0.003), (128, 300, 128, 1, 3e-4),
    (128, 300, 128, 1, 0), (128, 300, 128, 2, 0), (128, 256, 2, 1, 0), (128, 256, 4, 1, 0), (200, 500, 8, 1, 0), (200, 500, 8, 2, 1e-4),
    (500, 200, 400, 1, 0), (300, 300, 300, 30, 1e-3), (1000, 512, 4, 1, 0), (512, 4608, 512, 1, 0), (768, 768, 8, 2, 0), (1250, 1250, 2, 1, 1e-3),
    (2090, 1368, 16, 1, 0), (2500, 2500, 2500, 2, 0)])
def test_low_rank_and_few_rows(m, n, live, rank, noise):
    _check(_few_rows(m, n, live, rank, noise, m + n + live), TOL)


@pytest.mark.parametrize("m,n", [(100, 256), (1000, 512), (130, 3000)])
def test_the_gradient_of_one_sample(m, n):
    _check(_one_sample(m, n, m), TOL)


@pytest.mark.parametrize("m,n,rank,noise", [(2, 2100, 1, 0), (2, 2100, 1, 0.01), (8, 3000, 1, 0.003), (2100, 5, 2, 0), (64, 2049, 1, 0), (1, 5000, 1, 0)])
def test_long_matrices_of_few_rows(m, n, rank, noise):
    """A shorter side of at most 64 and a longer one above 2048: the general form."""
    _check(_few_rows(m, n, m, rank, noise, n), TOL)


def test_a_batch_of_matrices_of_unlike_rank():
    u = torch.stack([_few_rows(256, 300, live, rank, 0, live) for live, rank in ((1, 1), (2, 1), (256, 1), (256, 3), (256, 256), (17, 4))])
    _check(u, TOL, batch=6)


@pytest.mark.parametrize("steps", [1, 2, 3, 4])
def test_fewer_steps(steps):
    """Which halves of X a step takes depends on how many steps there are."""
    u = _few_rows(200, 500, 4, 1, 0, steps)
    got = OrthUpdate(200, 500, steps=steps).update(u, out_dtype=F32)[0]
    assert _off(got, _exact(u, steps)) < TOL


@pytest.mark.parametrize("m,n,live,rank,noise", [(64, 152, 64, 1, 0), (64, 324, 64, 1, 1e-4), (64, 576, 2, 1, 0), (2, 36, 2, 1, 0), (2, 2048, 2, 1, 0),
                                                 (48, 48, 8, 2, 1e-4), (1024, 16, 300, 1, 0)])
def test_small_matrices_of_low_rank(m, n, live, rank, noise):
    _check(_few_rows(m, n, live, rank, noise, m + n), TOL_SMALL)


@pytest.mark.parametrize("m,n,tol", [(128, 300, TOL), (48, 100, TOL_SMALL)])
@pytest.mark.parametrize("coef,steps,largest,b_largest", [((1.98, 0.0, 0.0), 4, 7.77, 0), ((1.72, 0.0, 1.0), 2, 2.73, 55)])
def test_coefficients_near_the_documented_limits(m, n, tol, coef, steps, largest, b_largest):
    """Equal entries: the one singular value is 1 at first.  The first coefficients take it to 7.76 before the last step (A up to 60.3), the
    second to 2.72, where B is 54.7; results are finite and as exact as elsewhere."""
    s = 1.0
    for _ in range(steps - 1):
        s *= coef[0] + coef[1] * s ** 2 + coef[2] * s ** 4
    assert 0.99 * largest < s < largest < 8 and coef[1] * s ** 2 + coef[2] * s ** 4 <= b_largest < 64
    u = torch.ones(m, n, device="cuda")
    got = OrthUpdate(m, n, steps=steps, coef=coef).update(u, out_dtype=F32)[0]
    assert torch.isfinite(got).all()
    assert _off(got, _exact(u, steps, coef)) < tol


@pytest.mark.parametrize("m,n", [(80, 120), (300, 140), (40, 72)])
@pytest.mark.parametrize("sigma,eps", [(1e-44, 0.0), (1e-41, 0.0), (1e-38, 0.0), (1e-36, 0.0), (2e36, 0.0), (5e37, 0.0), (5e37, 1e-7)])
def test_norms_outside_32_bits(m, n, sigma, eps):
    """1024 / norm passes the largest float below a norm of 3e-36, the norm itself from 3.4e38 on; the entries are finite and so is the
    update.  Tolerance: that of ordinary inputs, 2e-3."""
    g = torch.randn(m, n, device="cuda", generator=_gen(m)) + 0.2
    g = g.clamp(-5, 5) * sigma
    assert torch.isfinite(g).all() and (g != 0).any()
    got = OrthUpdate(m, n, eps=eps).update(g, out_dtype=F32)[0]
    assert _off(got, _exact(g, eps=eps)) < 2e-3

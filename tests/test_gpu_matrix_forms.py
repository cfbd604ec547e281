"""Every form in which a product is taken (single CTAs with tiles of 64, 128, 192 and 256 columns, clusters of 2, 4 and 8 that split K, pairs of
CTAs with and without halved last tiles), reached by its size: plan_mma chooses by fitted times, so the sizes are those at which each is chosen
on a device of 148 SMs, with ragged ones beside them."""
import pytest
import torch

from paper_1905_05957_b200 import Int8Linear, Int8Matrix, OrthUpdate, int8_matmul, int8_quantize
from paper_1905_05957_b200.matrix_ops import device_status

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16
U32 = 2.0 ** -24
COEF = (3.4445, -4.7750, 2.0315)


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _codes(rows, cols, seed):
    g = _gen(seed)
    q = torch.randint(-127, 128, (rows, cols), device="cuda", generator=g, dtype=torch.int8)
    return Int8Matrix.pack(q, torch.rand(rows, device="cuda", generator=g) + 0.5)


I8_FORMS = [
    (1000, 1200, 1000),                              # 128 columns
    (1200, 2048, 2048), (1201, 2049, 2047),          # 192
    (1800, 2048, 2048), (1799, 2047, 2049),          # 256
    (400, 1200, 16384), (400, 640, 8192), (400, 200, 8192), (399, 641, 8191),            # 128, K split by 2, 4, 8
    (1200, 400, 8192), (300, 400, 8192), (65, 65, 4096), (299, 401, 8190),               # 64, split
    (1536, 3000, 16384), (3000, 4096, 4096), (1536, 1536, 4096), (4096, 2500, 2048),     # pairs: whole tiles, rounds, halves, both
    (1535, 3001, 8190), (2999, 4095, 4097), (4095, 2501, 2050),
]


@pytest.mark.parametrize("m,n,k", I8_FORMS)
def test_8_bit_products(m, n, k):
    a, b = _codes(m, k, 1), _codes(n, k, 2)
    bias = torch.randn(n, device="cuda", generator=_gen(3)) * 100 if n % 2 else None
    # 32-bit results whose rows start on 32 bytes, and on no boundary (operands exchanged)
    ld = (n + 7) // 8 * 8
    store = torch.full((m, ld), -7.0, device="cuda")
    y = int8_matmul(a, b, bias, out=store[:, :n])
    s = a.codes.double() @ b.codes.double().T          # whole numbers below 2^53: exact
    plain = s * a.scale.double()[:, None] * b.scale.double()
    want = plain if bias is None else plain + bias.double()
    # conversion of the sum, two multiplications, one addition
    assert ((y.double() - want).abs() <= 3.01 * U32 * plain.abs() + 2.01 * U32 * want.abs() + 1e-30).all()
    assert (store[:, n:] == -7).all()
    odd = torch.full((m, ld + 9), -7.0, device="cuda")
    assert torch.equal(int8_matmul(a, b, bias, out=odd[:, 3:3 + n]), y)
    assert (odd[:, :3] == -7).all() and (odd[:, 3 + n:] == -7).all()
    half = torch.empty(m, (n + 15) // 16 * 16, dtype=BF16, device="cuda")[:, :n]
    assert torch.equal(int8_matmul(a, b, bias, out=half), y.to(BF16))
    assert device_status() == 0


def test_a_large_layer_in_training():
    """Forward and both gradients by pairs; each equals the product of its codes."""
    x, w = (torch.randn(2048, 4096, device="cuda", generator=_gen(s)).to(BF16) for s in (1, 2))
    dy = torch.randn(2048, 2048, device="cuda", generator=_gen(3)).to(BF16)
    layer = Int8Linear(w)
    y = layer.forward(x, training=True)
    dx, dw, _ = layer.backward(dy)

    def product(a, b, dtype):
        s = a.codes.double() @ b.codes.double().T
        return (s.float() * a.scale[:, None] * b.scale).to(dtype)

    rows, cols = (lambda v: int8_quantize(v)), (lambda v: int8_quantize(v, rows=False, cols=True))
    assert torch.equal(y, product(rows(x), rows(w), BF16))
    assert torch.equal(dx, product(rows(dy), cols(w), BF16))
    assert torch.equal(dw, product(cols(dy), cols(x), F32))


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows,cols", [(3, 8192), (3, 8196), (5, 16384), (5, 16392), (4, 28672), (2, 131072), (3, 20002), (2, 40)])
def test_codes_of_long_rows(dtype, rows, cols):
    """Rows on 16-byte boundaries below and above what a CTA keeps in registers, and with ends of less than 16 bytes: the formula in 32 bits,
    one operation at a time."""
    x = (torch.randn(rows, cols, device="cuda", generator=_gen(cols)) * 3).to(dtype)
    ld = (cols + 7) // 8 * 8
    store = torch.full((rows, ld), 1e30, device="cuda").to(dtype)      # what lies between the rows is in no maximum
    store[:, :cols] = x
    v = x.float()
    s = v.abs().amax(1) * torch.tensor(1 / 127, dtype=F32, device="cuda")
    q = torch.round(v * torch.reciprocal(s)[:, None])
    for given in (x, store[:, :cols]):
        got = int8_quantize(given)
        assert torch.equal(got.scale, s) and torch.equal(got.codes.float(), q)


def _exact(u, steps=5, coef=COEF, eps=1e-7):
    x = u.double()
    tall = x.shape[-2] > x.shape[-1]
    x = x.mT if tall else x
    x = x / (x.square().sum((-2, -1), keepdim=True).sqrt() + eps)
    for _ in range(steps):
        a = x @ x.mT
        x = coef[0] * x + (coef[1] * a + coef[2] * a @ a) @ x
    return x.mT if tall else x


# batch, rows, columns: the forms of A = X X^T, of A A and of B X
ORTH_FORMS = [
    (1, 1800, 2500),                                   # 128; 128; pairs with halves
    (1, 768, 3000), (3, 200, 4096),                    # 128 split by 4 and by 8; 64; 128 and 64
    (3, 1200, 1200), (3, 1200, 1536),                  # 192; 256; 64 and pairs with halves
    (12, 640, 1536), (12, 768, 1200),                  # 256; 64 and 128; 128 and pairs in rounds
    (1, 1200, 4096), (12, 768, 3000),                  # 64; 64; pairs with halves; 256; 128; pairs in rounds
    (12, 200, 4096), (12, 65, 2500), (1, 65, 2048), (1, 4096, 65),      # 64 split by 2, 4 and 8
    (12, 1000, 2500), (12, 400, 4096), (1, 1800, 3000), (12, 1200, 1200),     # pairs: rounds, halves, both
    (3, 1000, 1000), (3, 512, 4608), (12, 768, 768),   # 128; 128; 192
    (3, 1800, 3000), (3, 3000, 1800), (1, 2048, 2500), (1, 4096, 4096),       # A A by pairs: halves, then rounds
    (1, 512, 2500), (1, 640, 4096), (1, 1000, 4096),   # B X with 128, 192 and 256 columns
    (1, 64, 2049), (2, 40, 5000), (3, 5000, 17),       # a shorter side of at most 64 in the general form
    (1, 1799, 2501), (12, 399, 4095), (3, 1201, 1535), (1, 2047, 2501), (3, 513, 4607),     # the same, ragged
]


@pytest.mark.parametrize("batch,m,n", ORTH_FORMS)
def test_updates(batch, m, n):
    """Strong directions and noise of a tenth: the errors of ordinary updates, 2e-3 (each of three operands of 11 bits a step off by 2^-12,
    five steps: sqrt(15) 2^-12 = 1e-3, doubled for what grows).  On a workspace of NaN: what is read was written."""
    g = _gen(m + n)
    r = max(1, min(m, n) // 8)
    u = torch.randn(batch, m, r, device="cuda", generator=g) @ torch.randn(batch, r, n, device="cuda", generator=g) / r ** 0.5
    u = u + 0.1 * torch.randn(batch, m, n, device="cuda", generator=g)
    plan = OrthUpdate(m, n, batch=batch)
    plan.workspace.fill_(0xFF)
    got = plan.update(u, out_dtype=F32)
    for i in range(batch):
        want = _exact(u[i])
        assert float((got[i].double() - want).norm() / want.norm()) < 2e-3
    assert torch.equal(plan.update(u, out_dtype=BF16), got.to(BF16))
    x = torch.ones_like(u)
    plan.update(u, out_dtype=None, x=x, gamma=0.5)
    scale = max(1.0, m / n) ** 0.5
    assert ((x - (1 - 0.5 * scale * got)).abs() <= 4 * 2.0 ** -24 * (2 + scale * got.abs())).all()
    assert not plan.timed_out()

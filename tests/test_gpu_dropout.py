"""Dropout against a mask drawn by the oracle's generator: every value has one right answer."""
import math

import numpy as np
import pytest
import torch

import oracle
from paper_1905_05957_b200 import DsqError, dropout

pytestmark = pytest.mark.gpu
TYPES = [torch.float32, torch.bfloat16, torch.float16]


def kept(rows, cols, p, seed, step, layer):
    """The mask, one call of the oracle's Philox4x32-10 for every eight entries."""
    key = np.array([seed & 0xFFFFFFFF, (seed >> 32 & 0xFFFFFFFF) ^ 0x44524F50], dtype=np.uint32)
    half = np.zeros((rows, -(-cols // 8), 8), dtype=np.uint32)
    for r in range(rows):
        for g in range(half.shape[1]):
            w = oracle.philox4x32_10(np.array([g, r, layer, step], dtype=np.uint32), key)
            half[r, g, 0::2], half[r, g, 1::2] = w & 0xFFFF, w >> 16
    return torch.from_numpy(half.reshape(rows, -1)[:, :cols] >= math.floor(p * 65536 + 0.5)).cuda()


def _x(rows, cols, dtype, seed=1):
    return torch.randn(rows, cols, device="cuda", generator=torch.Generator(device="cuda").manual_seed(seed)).to(dtype)


def expected(x, p, mask):
    scale = torch.tensor(65536 / (65536 - math.floor(p * 65536 + 0.5)), dtype=torch.float32, device="cuda")
    return torch.where(mask, x.float() * scale, torch.zeros((), device="cuda")).to(x.dtype)      # one product in 32 bits, rounded


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 8), (3, 7), (5, 9), (64, 48), (33, 130), (7, 2056), (300, 33), (2, 4099)])
def test_values(rows, cols, dtype):
    x = _x(rows, cols, dtype)
    for p, seed, step, layer in ((0.1, 5, 0, 0), (0.5, (7 << 32) + 11, 3, 2), (0.9, 2 ** 64 - 1, 2 ** 32 - 1, 2 ** 32 - 1)):
        assert torch.equal(dropout(x, p, seed, step=step, layer=layer), expected(x, p, kept(rows, cols, p, seed, step, layer)))


@pytest.mark.parametrize("dtype", TYPES)
def test_rows_within_wider_rows_and_in_place(dtype):
    mask = kept(20, 50, 0.3, 9, 0, 0)
    for pad, offset in ((14, 0), (3, 1), (0, 5)):
        buf = torch.full((offset + 20 * (50 + pad) + 32,), 3.0, dtype=dtype, device="cuda")
        x = buf.as_strided((20, 50), (50 + pad, 1), offset)
        x.copy_(_x(20, 50, dtype))
        want = expected(x, 0.3, mask)
        assert torch.equal(dropout(x, 0.3, 9), want)
        assert dropout(x, 0.3, 9, out=x) is x and torch.equal(x, want)
        x.fill_(3.0)
        assert bool((buf == 3.0).all())      # nothing beside it was written


def test_columns_in_any_layout():
    x = _x(40, 30, torch.float32)
    assert torch.equal(dropout(x.t().contiguous().t(), 0.2, 1), dropout(x, 0.2, 1))


def test_many_rows():
    """More rows than a grid has, the last ones among them."""
    rows = 300_000
    x = torch.ones(rows, 3, device="cuda")
    y = dropout(x, 0.25, 4)
    key = np.array([4, 0x44524F50], dtype=np.uint32)
    for r in (0, 1, 32767, 32768, 131071, 262144, rows - 1):
        w = oracle.philox4x32_10(np.array([0, r, 0, 0], dtype=np.uint32), key)
        want = [h >= 16384 for h in (int(w[0]) & 0xFFFF, int(w[0]) >> 16, int(w[1]) & 0xFFFF)]
        assert (y[r] != 0).tolist() == want
    n = y.numel()
    assert abs(int((y == 0).sum()) - n / 4) < 5 * math.sqrt(n * 3 / 16)      # five standard deviations


def test_what_is_dropped_is_zero_whatever_it_was():
    x = torch.full((64, 64), float("nan"), device="cuda")
    x[32:] = float("inf")
    mask = kept(64, 64, 0.5, 3, 0, 0)
    y = dropout(x, 0.5, 3)
    assert bool((y[~mask] == 0).all()) and bool(y[:32][mask[:32]].isnan().all()) and bool(y[32:][mask[32:]].isinf().all())


def test_nothing_dropped_and_nothing_there():
    x = _x(10, 10, torch.bfloat16)
    assert torch.equal(dropout(x, 0.0, 1), x) and torch.equal(dropout(x, 1e-6, 1), x)
    assert dropout(x[:0], 0.5, 1).shape == (0, 10) and dropout(x[:, :0], 0.5, 1).shape == (10, 0)


def test_draws_differ_and_repeat():
    x = torch.ones(100, 1000, device="cuda")
    first = dropout(x, 0.5, 1)
    assert torch.equal(first, dropout(x, 0.5, 1))
    for kw in (dict(seed=2), dict(seed=1 + (1 << 32)), dict(seed=1, step=1), dict(seed=1, layer=1)):
        same = float((dropout(x, 0.5, **kw) == first).float().mean())
        assert abs(same - 0.5) < 5 * 0.5 / math.sqrt(x.numel())


def test_refusals():
    x = _x(10, 16, torch.bfloat16)
    for p in (-0.1, 1.0, 1.5, float("nan"), 1 - 1e-6):
        with pytest.raises(ValueError):
            dropout(x, p, 1)
    for kw in (dict(step=-1), dict(layer=1 << 32), dict(out=x[:9])):
        with pytest.raises(ValueError):
            dropout(x, 0.1, 1, **kw)
    with pytest.raises(TypeError):
        dropout(x.double(), 0.1, 1)
    with pytest.raises(TypeError):
        dropout(x, 0.1, 1, out=x.float())
    with pytest.raises(ValueError):
        dropout(x.cpu(), 0.1, 1)
    with pytest.raises(ValueError):
        dropout(x[0], 0.1, 1)
    with pytest.raises(DsqError):
        dropout(x[:9], 0.1, 1, out=x[1:])      # over its input, a row off


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,cols", [(5, 8), (33, 131), (300, 2056)])
def test_columns_of_one_buffer(rows, cols, dtype):
    """Input and output side by side in wider rows; what does share memory is refused."""
    buf = torch.zeros(rows, 2 * cols, device="cuda", dtype=dtype)
    x, out = buf[:, :cols], buf[:, cols:]
    x.copy_(_x(rows, cols, dtype))
    want = dropout(x.clone(), 0.3, 5)
    dropout(x, 0.3, 5, out=out)
    assert torch.equal(out, want) and torch.equal(x, _x(rows, cols, dtype))
    with pytest.raises(DsqError):
        dropout(x, 0.3, 5, out=buf[:, cols - 1:2 * cols - 1])

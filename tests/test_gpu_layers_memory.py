"""Memory that layers and joints use without owning it: parameters whose storage is replaced between calls."""
import pytest
import torch

from paper_1905_05957_b200 import ResidualNorm

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

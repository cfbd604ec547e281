"""Memory that the matrix operators own and streams other than the one it was allocated on: what is dropped before the stream has run may
not be handed out again until it has."""
import pytest
import torch

from paper_1905_05957_b200 import OrthUpdate

pytestmark = pytest.mark.gpu


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _behind():
    """A stream with some milliseconds of work before whatever comes next."""
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        busy = torch.randn(4096, 4096, device="cuda")
        for _ in range(40):
            busy = torch.sin(busy)
    return s


def _overwrite(sizes):
    """Allocations of these many bytes on the current stream, filled with what would be NaN in any type."""
    for _ in range(4):
        held = [torch.full((n,), 0xFF, dtype=torch.uint8, device="cuda") for n in sizes]
        del held


@pytest.mark.parametrize("m,n", [(300, 500), (1000, 512), (40, 72)])
def test_a_plan_dropped_before_its_stream_has_run(m, n):
    g = torch.randn(m, n, device="cuda", generator=_gen(m))
    buf0 = torch.randn(m, n, device="cuda", generator=_gen(n))
    keep = OrthUpdate(m, n)
    want_buf, x0 = buf0.clone(), torch.randn(m, n, device="cuda", generator=_gen(3))
    want_x = x0.clone()
    want = keep.update(g, want_buf, out_dtype=torch.float32, x=want_x, gamma=0.1)
    sizes = (keep.workspace.numel(), keep.workspace.numel() // 2, 512, 16)
    buf, x, out = buf0.clone(), x0.clone(), torch.empty(m, n, device="cuda")
    torch.cuda.synchronize()
    plan = OrthUpdate(m, n)
    s = _behind()
    plan.update(g, buf, out=out, x=x, gamma=0.1, stream=s)
    del plan
    _overwrite(sizes)
    torch.cuda.synchronize()
    assert torch.equal(out, want[0]) and torch.equal(buf, want_buf) and torch.equal(x, want_x)

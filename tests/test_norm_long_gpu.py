"""Group norm on stretches so long that a CTA reads them through its ring of shared memory many times over:
the same tolerances as for the other sizes."""
import pytest
import torch

from paper_2003_06513_gb300 import norm
from test_norm_gpu import DT, _check_backward, _check_forward, _inputs, _tensor

pytestmark = pytest.mark.gpu

# n, c, g, h, w; type; activation: whole vectors in a group; vectors across groups; one channel a vector; groups
# of more channels than a CTA has threads; stretches that end inside a round
FORWARD = [((9, 64, 32, 200, 211), "f32", "relu"), ((10, 312, 8, 120, 131), "f16", "silu"), ((4, 75, 5, 300, 301), "bf16", "none"),
           ((2, 1024, 2, 110, 109), "f32", "silu")]
BACKWARD = [((16, 128, 32, 112, 113), "f16", "silu"), ((4, 75, 5, 300, 301), "bf16", "relu"), ((2, 1024, 2, 110, 109), "f32", "none"),
            ((5, 312, 8, 120, 131), "f16", "relu")]


def _streamed_in_rounds(shape, dtype, backward):
    n, c, g, h, w = shape
    align = 16
    while c * (4 if dtype == "f32" else 2) % align:
        align //= 2
    p = norm.plan((n, c, h, w), g, DT[dtype], backward, align)
    return p["path"] == 1 and p["pixels"] * p["columns"] > 1.5 * p["held"]


@pytest.mark.parametrize("shape,dtype,kind", FORWARD, ids=str)
def test_forward(shape, dtype, kind):
    n, c, g, h, w = shape
    assert _streamed_in_rounds(shape, dtype, False)
    x, ga, be = _inputs((n, c, h, w), dtype, c)
    t = _tensor(x, dtype)
    y, _, _ = _check_forward(x, t, g, ga, be, kind, dtype)
    over, _, _ = norm.pp_group_norm(t, g, torch.from_numpy(ga).cuda(), torch.from_numpy(be).cuda(), 1e-5, kind, out=t)
    assert over.data_ptr() == t.data_ptr() and torch.equal(over, y)


@pytest.mark.parametrize("shape,dtype,kind", BACKWARD, ids=str)
def test_backward(shape, dtype, kind):
    n, c, g, h, w = shape
    assert _streamed_in_rounds(shape, dtype, True)
    x, ga, be = _inputs((n, c, h, w), dtype, c + 1)
    dy, _, _ = _inputs((n, c, h, w), dtype, c + 2)
    first = _check_backward(x, dy, _tensor(x, dtype), _tensor(dy, dtype), g, ga, be, kind, dtype)
    again = _check_backward(x, dy, _tensor(x, dtype), _tensor(dy, dtype), g, ga, be, kind, dtype)
    assert all(torch.equal(a, b) for a, b in zip(first, again))

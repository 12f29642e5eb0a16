"""Group norm on stretches so long that a CTA reads them through its ring of shared memory many times over:
the same tolerances as for the other sizes."""
import os
import subprocess
import sys

import pytest
import torch

from conftest import ROOT
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


_DIGESTS = """
import hashlib, torch
from paper_2003_06513_gb300 import norm
gen = torch.Generator(device="cuda").manual_seed(3)
for n, c, h, w, g in ((2, 32, 28, 28, 8), (8, 64, 224, 224, 32)):
    x, dy = (torch.randn(n, c, h, w, generator=gen, device="cuda").contiguous(memory_format=torch.channels_last) for _ in range(2))
    y, mean, rstd = norm.pp_group_norm(x, g, act="silu")
    got = (y, mean, rstd) + tuple(norm.pp_group_norm_backward(dy, x, mean, rstd, g, act="silu"))
    print(*[hashlib.sha256(t.cpu().numpy().tobytes()).hexdigest() for t in got])
"""


def test_plain_launches_give_the_same_bits():
    """PATCONV_PDL=0, read once a process: every kernel waits for the end of the one before it."""
    assert norm.plan((2, 32, 28, 28), 8)["path"] == 2 and norm.plan((8, 64, 224, 224), 32)["path"] == 1

    def digests(**env):
        run = subprocess.run([sys.executable, "-c", _DIGESTS], env={**os.environ, **env}, cwd=ROOT, capture_output=True,
                             text=True, timeout=300)
        assert run.returncode == 0, run.stderr
        return run.stdout.split()
    early, plain = digests(PATCONV_PDL="1"), digests(PATCONV_PDL="0")
    assert len(early) == 12 and early == plain

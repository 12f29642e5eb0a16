"""The group norm's plans (host only): which form a call takes, and that a plan covers the call and fits an SM."""
import math

import pytest
import torch

from paper_2003_06513_gb300 import norm

SHAPES = [((1, 64, 32, 32), 8), ((32, 256, 56, 56), 32), ((32, 64, 224, 224), 32), ((5, 150, 61, 45), 10),
          ((32, 512, 14, 14), 32), ((32, 128, 112, 112), 32), ((64, 960, 7, 7), 32), ((1, 1, 1, 1), 1),
          ((2, 7, 3, 5), 7), ((1, 4096, 1, 1), 1), ((3, 24576, 2, 2), 8), ((1, 1, 1000, 1000), 1)]


@pytest.mark.parametrize("backward", [False, True])
@pytest.mark.parametrize("dtype", [torch.float32, torch.float16, torch.bfloat16])
@pytest.mark.parametrize("shape,groups", SHAPES)
def test_plans_cover_the_call_and_fit(shape, groups, dtype, backward):
    n, c, h, w = shape
    size = 4 if dtype == torch.float32 else 2
    for align in (size, 4, 8, 16):
        if align < size:
            continue
        p = norm.plan(shape, groups, dtype, backward, align)
        assert c % p["channels"] == 0 and p["channels"] * size <= align
        slab = p["columns"] * p["channels"]
        stretches = math.ceil(h * w / p["pixels"])
        vector = p["channels"] * size * (2 if backward else 1)
        assert p["held"] * vector <= 160 * 1024
        if p["path"] == 2:                       # whole groups, one cluster a sample's slab, all of it held
            assert p["pixels"] * p["columns"] <= p["held"]
            assert slab % (c // groups) == 0 and c % slab == 0 and slab <= 1024
            assert stretches <= p["cluster"] in (1, 2, 4, 8)
            assert p["ctas"] == n * (c // slab) * p["cluster"]
        else:
            assert p["path"] == 1 and p["cluster"] == 0
            assert p["ctas"] == n * stretches * math.ceil(c / slab)


def test_both_forms_are_taken():
    taken = {(norm.plan(s, g, dt, b)["path"], b) for s, g in SHAPES for dt in (torch.float32, torch.float16)
             for b in (False, True)}
    assert taken == {(1, False), (2, False), (1, True), (2, True)}


def test_units_that_no_cluster_holds_are_streamed():
    assert norm.plan((32, 64, 224, 224), 1)["path"] == 1
    assert norm.plan((1, 8192, 1, 1), 1)["path"] == 1          # a group wider than a CTA's vectors

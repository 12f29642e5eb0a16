"""The distillation loss on the GPU at the edges of its arguments: parts of weight 0 beside what is not finite."""
import math

import numpy as np
import pytest
import torch

from paper_2003_06513_gb300 import distill

pytestmark = pytest.mark.gpu

# a row a warp, a CTA, several CTAs
SIZES = [(1300, 60, 5), (6, 50, 4), (7, 3000, 40), (2, 70001, 33)]


def _case(rows, classes, k, seed):
    rng = np.random.default_rng(seed)
    s = torch.from_numpy(rng.standard_normal((rows, classes)) * 2).float().cuda()
    teacher = torch.from_numpy(rng.standard_normal((rows, classes)) * 2).float().cuda()
    return s, distill.pp_top_logits(teacher, k, 2.0), torch.from_numpy(rng.integers(0, classes, rows)).cuda()


def _both(s, top, y, alpha, g, rest=True):
    args = (top.values, top.indices, top.rest if rest else None, y, 2.0, alpha)
    loss, stats = distill.pp_distill(s, *args)
    return loss, distill.pp_distill_backward(g, s, stats, *args)


@pytest.mark.parametrize("rest", [False, True])
@pytest.mark.parametrize("rows,classes,k", SIZES)
def test_a_teacher_of_no_weight_is_not_looked_at(rows, classes, k, rest):
    """alpha 0 beside a teacher's logit or rest that is NaN or infinite: the labels' loss and gradient, to the bit."""
    s, top, y = _case(rows, classes, k, 1)
    g = torch.rand(rows, device="cuda") + 0.5
    want = _both(s, top, y, 0.0, g, rest)
    nothing = distill.TopLogits(top.values, torch.full_like(top.indices, -1), torch.full_like(top.rest, -math.inf))
    labels_alone = _both(s, nothing, y, 0.0, g, rest)
    assert torch.allclose(want[0], labels_alone[0], rtol=1e-5, atol=1e-5) and torch.allclose(want[1], labels_alone[1], rtol=1e-5, atol=1e-6)
    for bad in (math.inf, math.nan):
        for where in ("first", "last", "rest"):
            spoilt = distill.TopLogits(*(t.clone() for t in top))
            (spoilt.rest if where == "rest" else spoilt.values[:, 0 if where == "first" else k - 1])[1] = bad
            got = _both(s, spoilt, y, 0.0, g, rest)
            assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
            if rest or where != "rest":               # (with a weight it has its part)
                loss, d = _both(s, spoilt, y, 0.5, g, rest)
                assert torch.isnan(loss[1]) and torch.isnan(d[1]).any() and torch.isfinite(loss[0]) and torch.isfinite(d[0]).all()


@pytest.mark.parametrize("rest", [False, True])
@pytest.mark.parametrize("rows,classes,k", SIZES)
def test_a_row_of_parts_without_weight_has_no_gradient(rows, classes, k, rest):
    """A teacher beside alpha 0 and no label, a label beside alpha 1 and no teacher: loss and gradient are 0 whatever the row holds."""
    s, top, y = _case(rows, classes, k, 2)
    s[1, classes // 2], s[0, classes - 1] = math.nan, math.inf
    g = torch.rand(rows, device="cuda") + 0.5
    loss, d = _both(s, top, torch.full_like(y, -100), 0.0, g, rest)
    assert not loss.any() and not d.any()
    nothing = distill.TopLogits(top.values, torch.full_like(top.indices, -1), torch.full_like(top.rest, -math.inf))
    loss, d = _both(s, nothing, y, 1.0, g, rest)
    assert not loss.any() and not d.any()
    loss, d = _both(s, nothing, y, 0.5, g, rest)
    assert torch.isnan(loss[:2]).all() and torch.isnan(d[:2]).any(1).all() and torch.isfinite(loss[2:]).all()

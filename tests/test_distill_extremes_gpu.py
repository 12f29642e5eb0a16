"""The distillation loss on the GPU at the edges of its arguments: parts of weight 0 beside what is not finite, high temperatures
where student and teacher agree."""
import math

import numpy as np
import pytest
import torch

from oracle import distill as D
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


def _near(rng, rows, classes, k, t, gap, dtype):
    """(student, kept logits, their classes), fp64 values that the types hold: the student's kept logits are the teacher's but for a
    shift and 2^-9 T of noise; its other classes lie `gap` T below the least of them."""
    values = -np.sort(-rng.standard_normal((rows, k)) * 2, 1).astype(np.float32)
    at = np.argsort(rng.random((rows, classes)), 1)[:, :k]
    s = values.min(1, keepdims=True) - gap * t - rng.random((rows, classes)) * t
    np.put_along_axis(s, at, values + 0.75 + rng.standard_normal((rows, k)) * t * 2.0 ** -9, 1)
    return torch.from_numpy(s).to(dtype), values, at


def _bound(s, values, at, t, alpha):
    """(loss, bound of fp32's error) without `rest`, from a row's divergence D = sum p f(d) + o / Z: f(d) = e^d - 1 - d, d = log q - log p of the kept
    classes, o the mass of the classes that are not kept and Z that of all, relative to the largest logit.

    d = (x - m) / T - (u - max u) - log(Z / Zu): of the first term the difference, 1 / T and the product round, 3 U R / T; u and its
    maximum are products with 1 / T, 4 U V / T, and their difference rounds; the teacher's masses have exponents that are off by as much,
    exponentials by 4 U (2^-22) and 13 additions (256 values over 32 lanes); Z's are off by their exponents, 3 U a unit of
    (m - x) / T on the average over q, and by ``roundings``, n; the quotient, the logarithm (2 U of its size) and the last two differences
    round: |error of d| <= e = U (40 + 16 (R + 2 V) / T + 2 |log(Z / Zu)| + 3 mean) + n.

    Where D is small it is summed as it stands here.  f' = e^d - 1 is at most 1.3 |d| for |d| < 1/4, so p f is off by p (1.3 |d| e + e^2), and by
    p's own relative error, at most e, the series' ten roundings and 13 additions' of the sum; o is a sum of integers, off by its
    exponents, 4 U and 2^-53 a class.  Elsewhere the logarithms are summed: they are off by e, and their sum by its own roundings
    and p's relative error of their size."""
    x, v = np.take_along_axis(s, at, 1), values.astype(np.float64)
    m = s.max(1, keepdims=True)
    log_z, log_zu = D._lse((s - m) / t), D._lse((v - v.max(1, keepdims=True)) / t)
    p = (v - v.max(1, keepdims=True)) / t - log_zu[:, None]
    d, p = (x - m) / t - log_z[:, None] - p, np.exp(p)
    kept = np.zeros(s.shape, bool)
    np.put_along_axis(kept, at, True, 1)
    q = np.exp((s - m) / t - log_z[:, None])
    o = np.where(kept, 0.0, q).sum(1)
    far = np.where(kept, 0.0, m - s).max(1) / t
    n = D.roundings(s.shape[1])
    reach = (m - x).max(1) + 2 * np.abs(v).max(1)
    e = D.U * (40 + 16 * reach / t + 2 * np.abs(log_z - log_zu) + 3 * (q * (m - s)).sum(1) / t) + n
    f = (p * np.where(np.abs(d) < 0.25, np.expm1(d) - d, 0.0)).sum(1)
    fine = (p * (1.3 * np.abs(d) * e[:, None] + e[:, None] ** 2)).sum(1) + f * (e + 32 * D.U) + o * (e + D.U * (8 + 3 * far)) \
        + s.shape[1] * 2.0 ** -53 / np.exp(log_z)
    size = (p * ((v.max(1, keepdims=True) - v) + (x.max(1, keepdims=True) - x))).sum(1) / t
    plain = e + (size + (m - x.max(1, keepdims=True))[:, 0] / t) * (e + 16 * D.U)
    small = (f + o < (1 + size) / 512) & (np.abs(d).max(1) < 0.25)
    return alpha * t * t * (f + o), alpha * t * t * np.where(small, fine, fine + plain), np.abs(d).max(1) < 0.25


AGREE = [(64, 10, 10, 0.0), (3, 1, 1, 0.0), (5, 256, 256, 0.0), (1300, 30, 30, 0.0), (5, 300, 16, 5.0), (1300, 300, 16, 5.0), (4, 9000, 40, 12.0),
         (2, 70001, 33, 16.0), (6, 500, 20, 30.0), (1, 1048576, 100, 25.0)]


@pytest.mark.parametrize("dtype,t", [(torch.float32, 1.0), (torch.float32, 10.0), (torch.float32, 100.0), (torch.float32, 1000.0), (torch.float16, 1.0), (torch.float16, 10.0), (torch.float16, 100.0)])
@pytest.mark.parametrize("rows,classes,k,gap", AGREE)
def test_the_loss_where_student_and_teacher_agree(rows, classes, k, gap, dtype, t):
    """Without `rest`: the kept classes are all there are, or have nearly all of the student's mass.  The divergence is small beside its terms
    and the temperature's square is not."""
    rng = np.random.default_rng(classes + k)
    student, values, at = _near(rng, rows, classes, k, t, gap, dtype)
    s = student.double().numpy()
    want, tol, close = _bound(s, values, at, t, 0.8)
    assert np.isfinite(s).all() and close.all()
    np.testing.assert_allclose(want, D.distill(s, values, at, None, None, t, 0.8)[0], rtol=1e-6, atol=1e-12 * t * t)
    loss, _ = distill.pp_distill(student.cuda(), torch.from_numpy(values).cuda(), torch.from_numpy(at.astype(np.int32)).cuda(), None, None, t, 0.8)
    got = loss.double().cpu().numpy()
    worst = np.max(np.abs(got - want) / (tol + 4 * D.U * want + 1e-300))
    assert worst <= 1.0, f"{worst:.2f} times the tolerance"
    assert (got >= 0).all()


@pytest.mark.parametrize("t", [1.0, 100.0, 1000.0])
@pytest.mark.parametrize("rows,classes", [(64, 10), (5, 256), (1300, 30)])
def test_a_student_that_is_the_teacher_has_no_loss(rows, classes, t):
    """All classes kept, the same logits: the terms are squares of roundings."""
    s = torch.from_numpy(np.random.default_rng(3).standard_normal((rows, classes))).float()
    at = torch.arange(classes, dtype=torch.int32).expand(rows, classes).contiguous()
    loss, _ = distill.pp_distill(s.cuda(), s.cuda(), at.cuda(), None, None, t, 0.8)
    v = s.double().numpy()
    _, tol, _ = _bound(v, s.numpy(), at.long().numpy(), t, 0.8)
    assert (loss >= 0).all() and np.all(loss.double().cpu().numpy() <= tol)


@pytest.mark.parametrize("classes,k", [(12, 9), (3000, 40)])
def test_places_that_do_not_count_where_student_and_teacher_agree(classes, k):
    """Rows that are read a second time with empty places, kept logits of -inf (a class like any other that is not kept), a class given
    twice -- each place with half of its mass, the divergence of two such places is log(1/2) of it and below 0 -- and a label."""
    rng = np.random.default_rng(4)
    rows, t = 8, 10.0
    student, values, at = _near(rng, rows, classes, k, t, 14.0, torch.float32)
    s = student.double().numpy()
    at = at.astype(np.int64)
    spoilt, value = at.copy(), values.copy()
    spoilt[0, 1], spoilt[1, ::2], value[2, 3] = -1, classes + 7, -np.inf
    # the first class's mass in two halves, the last place's own class left to the others
    spoilt[3, k - 1] = spoilt[3, 0]
    value[3, 0] = value[3, k - 1] = values[3, 0] - t * math.log(2)
    y = at[:, 0].copy()
    want, _, _, size, _ = D.distill(s, value, spoilt, None, y, t, 0.8)
    loss, stats = distill.pp_distill(student.cuda(), torch.from_numpy(value).cuda(), torch.from_numpy(spoilt.astype(np.int32)).cuda(), None,
                                     torch.from_numpy(y).cuda(), t, 0.8)
    assert np.all(np.abs(loss.double().cpu().numpy() - want) <= D.roundings(classes) * size)
    clean, _, _ = _bound(s, values, at, t, 0.8)
    hard = D.distill(s, values, np.full_like(at, -1), None, y, t, 0.8)[0]
    rest = slice(4, None)
    _, tol, _ = _bound(s, values, at, t, 0.8)
    assert np.all(np.abs(loss.double().cpu().numpy() - clean - hard)[rest] <= (tol + 4 * D.U * (clean + hard) + D.U * 64 * (1 + hard))[rest])

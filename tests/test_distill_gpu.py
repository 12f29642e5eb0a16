"""A teacher's top logits, the distillation loss and its gradient on the GPU against the float64 oracle.  Tolerances are
numbers of fp32 roundings of the terms' sizes (oracle.distill.roundings) plus half a unit of the output type's last place."""
import math

import numpy as np
import pytest
import torch

from oracle import distill as D
from paper_2003_06513_gb300 import distill
from paper_2003_06513_gb300._lib import PatconvError

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
ULP = {"f32": (2.0 ** -24, 2.0 ** -120), "f16": (2.0 ** -11, 2.0 ** -25), "bf16": (2.0 ** -8, 2.0 ** -120)}


def _rows(rng, rows, classes, dtype, spread=2.5, wide=0, at=0):
    """Logits as the type holds them, on the host in fp64 and on the GPU, there as columns at .. of rows wider by ``wide``."""
    t = torch.from_numpy(rng.standard_normal((rows, classes)) * spread).to(DT[dtype])
    base = torch.full((rows, classes + wide), math.nan, dtype=DT[dtype], device="cuda")
    base[:, at:at + classes] = t.cuda()
    return t.double().numpy(), base[:, at:at + classes]


def _host(t):
    return t.detach().double().cpu().numpy()


# ------------------------------------------------------------------------------------- top logits

# rows, classes, k: one class; all kept; a row of a few values; around vectors, warps and CTAs; the most that is kept; few rows
# (a cluster has one); slices that do not fit shared memory
TOPS = [(1, 1, 1), (3, 5, 5), (4, 10, 4), (64, 10, 1), (5, 33, 32), (7, 100, 17), (2, 257, 256), (3, 1000, 16), (300, 1000, 256), (9, 1100, 256),
        (2, 4095, 31), (2, 4097, 33), (5, 21841, 50), (1, 50001, 1), (3, 65536, 256), (2, 200001, 200), (1, 1048576, 100), (320, 70001, 7)]


def _check_top(s, t, k, temperature=1.0):
    values, at, rest = D.top(s, k, temperature)
    got = distill.pp_top_logits(t, k, temperature)
    assert got.values.dtype == t.dtype and got.indices.dtype == torch.int32 and got.rest.dtype == torch.float32
    np.testing.assert_array_equal(got.indices.cpu().numpy(), at)
    np.testing.assert_array_equal(_host(got.values), values)
    # a sum of exponentials, whose exponents are rounded: the log is off by that many roundings, and by its own size's
    fine = np.isfinite(rest)
    np.testing.assert_array_equal(_host(got.rest)[~fine], rest[~fine])
    top = np.where(np.isfinite(s), np.abs(s), 0.0).max(1)
    tol = D.U * (64 + s.shape[1] / 128) + 4 * D.U * (np.abs(rest[fine]) + top[fine] / temperature)
    assert np.all(np.abs(_host(got.rest)[fine] - rest[fine]) <= tol)
    return got


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("shape", TOPS, ids=str)
def test_top(shape, dtype):
    rows, classes, k = shape
    rng = np.random.default_rng(classes + k)
    s, t = _rows(rng, rows, classes, dtype)
    _check_top(s, t, k, (1.0, 2.0, 3.5)[k % 3])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("wide,at", [(1, 0), (3, 1), (8, 8), (5, 5)])
def test_top_of_rows_of_a_wider_tensor(wide, at, dtype):
    for rows, classes, k in ((6, 1000, 20), (3, 30011, 60)):
        s, t = _rows(np.random.default_rng(1), rows, classes, dtype, wide=wide, at=at)
        _check_top(s, t, k)


@pytest.mark.parametrize("dtype", ["f32", "f16"])
@pytest.mark.parametrize("rows,classes,k", [(2, 700, 9), (2, 5000, 100), (1, 40000, 256), (400, 9000, 3)])
def test_top_where_many_are_equal(rows, classes, k, dtype):
    """The list of candidates runs over: equal rows, two values, few distinct values, -0 beside 0."""
    rng = np.random.default_rng(2)
    for s in (np.zeros((rows, classes)), np.where(rng.random((rows, classes)) < 0.5, 0.0, -0.0), rng.integers(0, 3, (rows, classes)).astype(float),
              np.full((rows, classes), -np.inf), np.where(rng.random((rows, classes)) < 0.001, 1.0, -np.inf)):
        _check_top(s, torch.from_numpy(s).to("cuda", DT[dtype]), k)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("classes,k", [(4096, 200), (32768, 64), (262144, 256)])
def test_top_where_the_large_ones_lie_together(classes, k, dtype):
    """Rising and falling rows, and large values in a few threads' places alone: bounds that many values reach."""
    rng = np.random.default_rng(3)
    wave = np.linspace(-5, 5, classes)
    few = rng.standard_normal(classes)
    few[np.arange(classes) // 8 % 512 == 3] += 100
    block = rng.standard_normal(classes)
    block[100:100 + min(classes // 2, 3000)] += 50
    s = torch.from_numpy(np.stack([wave, wave[::-1], few, block])).to(DT[dtype])
    _check_top(s.double().numpy(), s.cuda(), k)


def test_top_of_what_is_not_finite():
    s = np.random.default_rng(4).standard_normal((6, 2000)).astype(np.float32)
    s[0, [3, 1999]] = np.nan
    s[1, 77] = np.inf
    s[2, 5:] = -np.inf
    s[3, ::2] = -np.inf
    s[4, :] = np.inf
    s[5, :1500] = np.nan
    s[5, 7] = -np.nan
    t = torch.from_numpy(s).cuda()
    values, at, rest = D.top(s, 8, 1.0)
    got = distill.pp_top_logits(t, 8)
    np.testing.assert_array_equal(got.indices.cpu().numpy(), at)
    np.testing.assert_array_equal(_host(got.values), values)
    assert np.allclose(_host(got.rest)[[0, 1, 3]], rest[[0, 1, 3]], rtol=1e-6)
    assert float(got.rest[2]) == -math.inf and float(got.rest[4]) == math.inf and math.isnan(float(got.rest[5]))


# rows of few vectors with many kept, whose values themselves are counted; warps; one CTA of 128 to 512 threads; clusters for few rows
# and for many that would not stay in L2
FORMS = [(40, 200, 60), (40, 300, 128), (9, 520, 250), (300, 1000, 250), (5, 1500, 256), (7, 2047, 200), (1300, 60, 23), (1300, 130, 20),
         (1250, 2000, 23), (1250, 4000, 10), (64, 32768, 20), (3, 90000, 63), (20, 65536, 64), (330, 70001, 20), (160, 270001, 5)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape", FORMS, ids=str)
def test_top_in_every_form(shape, dtype):
    rows, classes, k = shape
    rng = np.random.default_rng(classes + k)
    s, t = _rows(rng, rows, classes, dtype, wide=3, at=2)
    _check_top(s, t, k, (1.0, 2.0, 3.5)[k % 3])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,classes,k", [(8, 300, 100), (8, 1000, 250), (1300, 100, 23), (8, 1500, 256)])
def test_top_of_short_rows_of_odd_values(rows, classes, k, dtype):
    """Equal values, hardly any that are not -inf, ones of very different size, rows of NaN but for few."""
    rng = np.random.default_rng(5)
    normal = rng.standard_normal((rows, classes))
    for s in (np.zeros((rows, classes)), rng.integers(-2, 2, (rows, classes)).astype(float), np.full((rows, classes), -np.inf),
              np.where(rng.random((rows, classes)) < 0.01, normal, -np.inf), normal * 10.0 ** rng.integers(-30, 30, (rows, classes)),
              -np.abs(normal), np.where(np.arange(classes) < k // 2, np.nan, normal)):
        t = torch.from_numpy(s).to(DT[dtype])
        _check_top(t.double().numpy(), t.cuda(), k, 1.0 if np.abs(np.nan_to_num(s, neginf=0.0)).max() < 10 else 1e3)


@pytest.mark.parametrize("classes,k", [(4800, 256), (8000, 250), (6000, 100)])
def test_top_of_rows_whose_others_are_hardly_less(classes, k):
    """One value in eight is 1, the seven beside it 0.9995: thousands of exponentials near 1."""
    s = torch.full((3, classes), 1 - 2.0 ** -11, dtype=torch.float16)
    s[:, ::8] = 1
    s[1] = s[1].flip(0)
    _check_top(s.double().numpy(), s.cuda(), k)


# ------------------------------------------------------------------------------------- the loss

# rows, classes, kept: a warp a row, a CTA, a cluster; kept 1, all, the most; odd sizes
SHAPES = [(1, 1, 1), (64, 10, 4), (5, 7, 7), (3, 255, 32), (3, 257, 256), (2000, 300, 20), (1300, 2048, 32), (1300, 2047, 33), (37, 1000, 16),
          (512, 1000, 16), (6, 5003, 100), (700, 3001, 50), (2, 65536, 256), (1, 262144, 64), (3, 200003, 31), (1, 1048576, 8)]


def _teacher(rng, rows, classes, k, dtype, empty=True):
    """Kept logits of random classes, some places empty, rows with none, a class given twice."""
    at = np.argsort(rng.random((rows, classes)), 1)[:, :k].astype(np.int64) if classes <= 4096 else \
        (np.arange(k)[None] * (classes // k) + rng.integers(0, classes // k, (rows, k)))[:, rng.permutation(k)]
    at = np.ascontiguousarray(at)
    values = torch.from_numpy(-np.sort(-rng.standard_normal((rows, k)) * 2 - 3, 1)).to(DT[dtype])
    rest = rng.standard_normal(rows).astype(np.float32) + 1
    if empty:
        at[rng.random((rows, k)) < 0.1] = -1
        at[rng.random(rows) < 0.1] = classes + 5
        if k > 1 and rows > 2:
            at[1, k - 1] = at[1, 0]
            at[2, :] = -1
            rest[2] = -np.inf
    return values.double().numpy(), at, rest, values.cuda(), torch.from_numpy(at.astype(np.int32)).cuda(), torch.from_numpy(rest).cuda()


def _within(got, want, tol, dtype, what):
    rel, small = ULP[dtype]
    fine = np.isfinite(want)
    np.testing.assert_array_equal(got[~fine], want[~fine], err_msg=what)
    tol = (tol + rel * (np.abs(want) + tol) + small)[fine]
    worst = np.max(np.abs(got[fine] - want[fine]) / tol) if fine.any() else 0.0
    assert worst <= 1.0, f"{what}: {worst:.2f} times the tolerance"


def _check(s, t, teacher, labels, temperature, alpha, rest, dtype, seed=0):
    values, at, r, dvalues, dat, dr = teacher
    drest, r = (dr, r) if rest else (None, None)
    dlabels = None if labels is None else torch.from_numpy(labels).cuda()
    want, wstats, wgrad, size, reach = D.distill(s, values, at, r, labels, temperature, alpha)
    loss, stats = distill.pp_distill(t, dvalues, dat, drest, dlabels, temperature, alpha)
    n = D.roundings(s.shape[1])
    _within(_host(loss), want, n * size, "f32", "loss")
    _within(_host(stats), wstats, n * np.abs(np.where(np.isfinite(wstats), wstats, 0)), "f32", "stats")
    g = np.random.default_rng(seed).standard_normal(s.shape[0]).astype(np.float32)
    g[-1:] = 0 if s.shape[0] > 1 else 1.5
    d = distill.pp_distill_backward(torch.from_numpy(g).cuda(), t, stats, dvalues, dat, drest, dlabels, temperature, alpha)
    assert d.shape == t.shape and d.dtype == t.dtype and d.is_contiguous()
    g = g.astype(np.float64)[:, None]
    _within(_host(d), g * wgrad, np.abs(g) * n * reach, dtype, "gradient")
    return loss, stats, d


def _labels(rng, rows, classes):
    y = rng.integers(0, classes, rows)
    y[rng.random(rows) < 0.2] = -100
    y[rng.random(rows) < 0.05] = classes
    return y


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_loss_and_gradient(shape, dtype):
    rows, classes, k = shape
    rng = np.random.default_rng(classes + k)
    s, t = _rows(rng, rows, classes, dtype)
    teacher = _teacher(rng, rows, classes, k, ("f32", "f16", "bf16")[k % 3])
    labels = _labels(rng, rows, classes) if k % 4 else None
    if labels is not None:
        labels[0] = max(0, min(classes - 1, int(teacher[1][0, 0])))         # the label among the kept
    for rest in (False, True):
        _check(s, t, teacher, labels, (1.0, 2.0, 3.5)[classes % 3], (0.5, 0.9, 1.0)[rows % 3], rest, dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape", [(1250, 4093, 20), (1250, 4096, 32), (1220, 8189, 9), (200, 66001, 30), (400, 65536, 5)], ids=str)
def test_loss_and_gradient_of_many_long_rows(shape, dtype):
    rows, classes, k = shape
    rng = np.random.default_rng(classes + k)
    s, t = _rows(rng, rows, classes, dtype, wide=1)
    _check(s, t, _teacher(rng, rows, classes, k, dtype), _labels(rng, rows, classes), 2.0, 0.7, True, dtype)


@pytest.mark.parametrize("labels", [False, True])
@pytest.mark.parametrize("rest", [False, True])
@pytest.mark.parametrize("temperature", [0.5, 1.0, 4.0])
@pytest.mark.parametrize("alpha", [0.0, 0.3, 1.0])
@pytest.mark.parametrize("rows,classes,k", [(40, 100, 9), (11, 3000, 40)])
def test_every_form(rows, classes, k, alpha, temperature, rest, labels):
    rng = np.random.default_rng(5)
    s, t = _rows(rng, rows, classes, "f32")
    teacher = _teacher(rng, rows, classes, k, "f32")
    _check(s, t, teacher, _labels(rng, rows, classes) if labels else None, temperature, alpha, rest, "f32")


@pytest.mark.parametrize("dtype", ["f32", "f16"])
@pytest.mark.parametrize("wide,at", [(1, 0), (3, 1), (8, 8), (5, 5), (16, 0)])
def test_rows_of_a_wider_tensor(wide, at, dtype):
    """Rows whose 16-byte boundaries lie elsewhere than those of the dense gradient; what lies beside them is not read."""
    for rows, classes, k in ((6, 1000, 20), (1500, 77, 5), (3, 30011, 60)):
        rng = np.random.default_rng(6)
        s, t = _rows(rng, rows, classes, dtype, wide=wide, at=at)
        _check(s, t, _teacher(rng, rows, classes, k, "f32"), _labels(rng, rows, classes), 2.0, 0.6, bool(wide % 2), dtype)


@pytest.mark.parametrize("classes", [50, 20000])
def test_where_the_kept_classes_have_nearly_all(classes):
    """The student's probability of the others is far below fp32's step at 1: it is summed, not subtracted."""
    rng = np.random.default_rng(7)
    rows, k = 9, 8
    s, _ = _rows(rng, rows, classes, "f32", 1.0)
    teacher = _teacher(rng, rows, classes, k, "f32", empty=False)
    np.put_along_axis(s, teacher[1], np.take_along_axis(s, teacher[1], 1) + 60.0, 1)
    s = s.astype(np.float32)
    _check(s.astype(np.float64), torch.from_numpy(s).cuda(), teacher, None, 1.0, 1.0, True, "f32")
    # and further down than an exponential of fp32 reaches
    np.put_along_axis(s, teacher[1], np.take_along_axis(s, teacher[1], 1) + 200.0, 1)
    _check(s.astype(np.float64), torch.from_numpy(s).cuda(), teacher, None, 1.0, 1.0, True, "f32")


@pytest.mark.parametrize("classes", [40, 9000])
def test_masked_classes(classes):
    """Logits of -inf or the type's lowest value: no probability, no gradient; a kept one of them makes the loss infinite."""
    rng = np.random.default_rng(8)
    rows, k = 6, 5
    s, _ = _rows(rng, rows, classes, "f32")
    teacher = _teacher(rng, rows, classes, k, "f32", empty=False)
    mask = rng.random((rows, classes)) < 0.7
    np.put_along_axis(mask, teacher[1], False, 1)
    s[:3][mask[:3]] = -np.inf
    s[3:5][mask[3:5]] = np.finfo(np.float32).min
    keep = np.zeros(classes, bool)
    keep[teacher[1][5]] = True
    s[5, ~keep] = -np.inf                                  # nothing but the kept ones is left
    t = torch.from_numpy(s.astype(np.float32)).cuda()
    s = t.double().cpu().numpy()
    y = teacher[1][:, 0].copy()
    _, _, d = _check(s, t, teacher, y, 2.0, 0.5, False, "f32")
    assert not d[torch.from_numpy(s <= -1e38).cuda()].any()
    values, at, r, dvalues, dat, dr = teacher
    r[5], dr[5] = -np.inf, -math.inf
    _check(s, t, teacher, y, 2.0, 0.5, True, "f32")
    s[0, at[0, 2]] = -np.inf
    loss, _ = distill.pp_distill(torch.from_numpy(s.astype(np.float32)).cuda(), dvalues, dat)
    assert math.isinf(float(loss[0])) and torch.isfinite(loss[1:]).all()


@pytest.mark.parametrize("temperature", [0.5, 2.0])
@pytest.mark.parametrize("classes", [40, 9000])
def test_rows_of_the_lowest_value(classes, temperature):
    """Nothing is left but the mask itself, and the lowest value times log2(e) is not in fp32's range: all classes are alike."""
    rng = np.random.default_rng(14)
    s = np.full((3, classes), float(np.finfo(np.float32).min))
    teacher = _teacher(rng, 3, classes, 5, "f32", empty=False)
    for rest in (False, True):
        _check(s, torch.from_numpy(s.astype(np.float32)).cuda(), teacher, np.array([3, -1, 7]), temperature, 0.5, rest, "f32")


@pytest.mark.parametrize("rest", [False, True])
def test_a_part_of_no_weight_takes_no_part(rest):
    """alpha 0 beside a kept class that the student's mask leaves out, alpha 1 beside such a label: infinite terms of weight 0."""
    rng = np.random.default_rng(20)
    for rows, classes in ((6, 50), (6, 5000)):
        s, t = _rows(rng, rows, classes, "f32")
        teacher = _teacher(rng, rows, classes, 4, "f32", empty=False)
        y = teacher[1][:, 1].copy()
        s[2, y[2]] = -np.inf
        t[2, y[2]] = -math.inf
        y[3] = -1
        _check(s, t, teacher, np.where(np.arange(rows) == 2, teacher[1][:, 0], y), 2.0, 0.0, rest, "f32")
        loss, stats = distill.pp_distill(t, teacher[3], teacher[4] * 0 - 1, None, torch.from_numpy(y).cuda(), 2.0, 1.0)
        assert not loss.any()


@pytest.mark.parametrize("rest", [False, True])
@pytest.mark.parametrize("rows,classes", [(30, 20), (5, 6000)])
def test_padded_rows_are_not_read(rows, classes, rest):
    """Rows without label and teacher, and rows whose loss has no gradient, hold NaN: zeros come out, and the others do not change."""
    rng = np.random.default_rng(9)
    s, t = _rows(rng, rows, classes, "f32")
    values, at, r, dvalues, dat, dr = _teacher(rng, rows, classes, 4, "f32", empty=False)
    y = torch.from_numpy(rng.integers(0, classes, rows)).cuda()
    drest = dr if rest else None
    g = torch.ones(rows, device="cuda")
    clean = distill.pp_distill(t, dvalues, dat, drest, y, 2.0, 0.5)
    dclean = distill.pp_distill_backward(g, t, clean[1], dvalues, dat, drest, y, 2.0, 0.5)
    spoilt = t.clone()
    spoilt[2] = math.nan
    spoilt[4] = math.inf
    y[2], dat[2] = -1, -1
    if rest:
        dr[2] = -math.inf
    g[4] = 0
    loss, stats = distill.pp_distill(spoilt, dvalues, dat, drest, y, 2.0, 0.5)
    d = distill.pp_distill_backward(g, spoilt, stats, dvalues, dat, drest, y, 2.0, 0.5)
    assert float(loss[2]) == 0 and not stats[2].any() and not d[2].any() and not d[4].any() and math.isnan(float(loss[4]))
    others = [i for i in range(rows) if i not in (2, 4)]
    assert torch.equal(loss[others], clean[0][others]) and torch.equal(d[others], dclean[others])


def test_what_is_not_finite_stays_in_its_row():
    rng = np.random.default_rng(10)
    s, t = _rows(rng, 5, 3000, "bf16")
    _, _, _, values, at, rest = _teacher(rng, 5, 3000, 4, "f32", empty=False)
    t[1, 17], t[3, 2999] = math.nan, math.inf
    loss, stats = distill.pp_distill(t, values, at, rest, None, 2.0, 1.0)
    d = distill.pp_distill_backward(torch.ones(5, device="cuda"), t, stats, values, at, rest, None, 2.0, 1.0)
    bad = torch.tensor([False, True, False, True, False], device="cuda")
    assert torch.equal(torch.isnan(loss), bad) and torch.equal(torch.isnan(d).any(1), bad)


@pytest.mark.parametrize("rows,classes", [(2000, 100), (3, 40000), (400, 1000)])
def test_in_place(rows, classes):
    rng = np.random.default_rng(11)
    _, t = _rows(rng, rows, classes, "f16")
    _, _, _, values, at, rest = _teacher(rng, rows, classes, 6, "f16")
    y = torch.from_numpy(_labels(rng, rows, classes)).cuda()
    g = torch.full((rows,), 0.25, device="cuda")
    _, stats = distill.pp_distill(t, values, at, rest, y, 2.0, 0.5)
    want = distill.pp_distill_backward(g, t, stats, values, at, rest, y, 2.0, 0.5)
    before = t._version
    got = distill.pp_distill_backward(g, t, stats, values, at, rest, y, 2.0, 0.5, out=t)
    assert got.data_ptr() == t.data_ptr() and t._version > before and torch.equal(got, want)


def test_nothing_to_do():
    s, at = torch.zeros(0, 9, device="cuda"), torch.zeros(0, 2, dtype=torch.int32, device="cuda")
    top = distill.pp_top_logits(s, 2)
    assert top.values.shape == (0, 2) and top.rest.shape == (0,)
    loss, stats = distill.pp_distill(s, s[:, :2], at)
    assert loss.shape == (0,) and distill.pp_distill_backward(loss, s, stats, s[:, :2], at).shape == (0, 9)


@pytest.mark.parametrize("rows,classes,k", [(1500, 300, 10), (40, 3000, 40), (2, 100000, 200)])
def test_the_same_bits_again_on_another_stream_and_in_a_graph(rows, classes, k):
    rng = np.random.default_rng(12)
    _, t = _rows(rng, rows, classes, "bf16")
    teacher = torch.from_numpy(rng.standard_normal((rows, classes))).to("cuda", torch.bfloat16)
    y = torch.from_numpy(_labels(rng, rows, classes)).cuda()
    g = torch.rand(rows, device="cuda")

    def all_of(**kw):
        top = distill.pp_top_logits(teacher, k, 2.0, **kw)
        loss, stats = distill.pp_distill(t, *top, y, 2.0, 0.5, **kw)
        return (*top, loss, stats, distill.pp_distill_backward(g, t, stats, *top, y, 2.0, 0.5, **kw))

    want = all_of()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    again, other = all_of(), all_of(stream=side)
    torch.cuda.synchronize()
    graph, second = torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = all_of()
    with torch.cuda.graph(second):
        captured2 = all_of()
    for _ in range(3):
        graph.replay()
        second.replay()
    torch.cuda.synchronize()
    for a in (again, other, captured, captured2):
        assert all(torch.equal(x, z) for x, z in zip(want, a))


def test_a_captured_training_step():
    """Selection, loss and gradient captured into a graph, replayed on other inputs."""
    g = torch.Generator("cuda").manual_seed(21)
    first, second = ([torch.randn(30, 2000, device="cuda", generator=g) * 2 for _ in range(2)] for _ in range(2))
    y = torch.randint(0, 2000, (30,), device="cuda", generator=g)

    def step(s, teacher):
        leaf = s.detach().requires_grad_(True)
        loss = distill.distill_loss(leaf, distill.pp_top_logits(teacher, 20, 2.0), y, 2.0, 0.5)
        return loss.detach(), torch.autograd.grad(loss.mean(), leaf)[0]

    want = step(*second)
    static = [t.clone() for t in first]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(*static)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step(*static)
    for t, new in zip(static, second):
        t.copy_(new)
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_autograd():
    """distill_loss's gradient is the formula's, for the mean over rows (one gradient for all) and for a sum with weights."""
    rng = np.random.default_rng(13)
    s, t = _rows(rng, 12, 500, "f32")
    values, at, r, dvalues, dat, dr = _teacher(rng, 12, 500, 9, "f32")
    y = _labels(rng, 12, 500)
    top = distill.TopLogits(dvalues, dat, dr)
    _, _, grad, _, reach = D.distill(s, values, at, r, y, 2.0, 0.7)
    w = torch.rand(12, device="cuda")
    for weights in (torch.full((12,), 1 / 12, device="cuda"), w):
        x = t.detach().clone().requires_grad_(True)
        loss = distill.distill_loss(x, top, torch.from_numpy(y).cuda(), 2.0, 0.7)
        (loss.mean() if weights is not w else (loss * w).sum()).backward()
        g = _host(weights)[:, None]
        _within(_host(x.grad), g * grad, (D.roundings(500) + 4 * D.U) * g * reach, "f32", "gradient")
    with torch.no_grad():
        assert not distill.distill_loss(x, top).requires_grad
    x = t.detach().clone().requires_grad_(True)
    both = distill.distill_loss(x, top, None, 2.0).sum() + distill.distill_loss(x, top, None, 1.0).sum()     # one leaf, two losses
    both.backward()
    want = D.distill(s, values, at, r, None, 2.0, 0.5), D.distill(s, values, at, r, None, 1.0, 0.5)
    _within(_host(x.grad), want[0][2] + want[1][2], (D.roundings(500) + 4 * D.U) * (want[0][4] + want[1][4]), "f32", "gradient of two")


def test_autograd_refuses_what_it_cannot_do():
    x = torch.randn(3, 40, device="cuda", requires_grad=True)
    top = distill.pp_top_logits(x.detach(), 4)
    loss = distill.distill_loss(x, top)
    with pytest.raises(RuntimeError, match="once"):
        torch.autograd.grad(loss.sum(), x, create_graph=True)
    with pytest.raises(PatconvError):
        distill.distill_loss(x, top, temperature=0.0)
    with pytest.raises(ValueError, match="labels"):
        distill.distill_loss(x, top, torch.zeros(3, device="cuda"))
    x.data.add_(1)
    loss = distill.distill_loss(x, top)
    with torch.no_grad():
        x.add_(1)                                       # what the gradient would be of has changed
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        loss.sum().backward()


def test_autograd_on_another_stream():
    x = torch.randn(50, 3000, device="cuda")
    top = distill.pp_top_logits(x, 9)
    want = x.clone().requires_grad_(True)
    distill.distill_loss(want * 0.5, top).sum().backward()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = x.clone().requires_grad_(True)
        distill.distill_loss(got * 0.5, top).sum().backward()
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(got.grad, want.grad)


def test_refusals():
    s = torch.zeros(4, 100, device="cuda")
    v, at, rest, y = s[:, :5].contiguous(), torch.zeros(4, 5, dtype=torch.int32, device="cuda"), torch.zeros(4, device="cuda"), torch.zeros(4, dtype=torch.long, device="cuda")
    for kw in (dict(k=0), dict(k=101), dict(k=5, logits=s.double()), dict(k=5, logits=s[0]), dict(k=5, logits=s.t()), dict(k=5, logits=s[:1].expand(4, 100)), dict(k=257, logits=torch.zeros(1, 300, device="cuda"))):
        with pytest.raises(ValueError):
            distill.pp_top_logits(**({"logits": s} | kw))
    with pytest.raises(PatconvError):
        distill.pp_top_logits(s, 5, 0.0)
    for kw in (dict(values=v[:3]), dict(values=v.double()), dict(values=s[:, :5]), dict(indices=at.long()), dict(indices=at[:, :4]), dict(rest=rest.half()),
               dict(rest=rest[:3]), dict(labels=y.int()), dict(labels=y[:3]), dict(labels=y.cpu()), dict(values=s, indices=torch.zeros(4, 100, dtype=torch.long, device="cuda"))):
        with pytest.raises(ValueError):
            distill.pp_distill(**({"logits": s, "values": v, "indices": at} | kw))
    for kw in (dict(temperature=0.0), dict(alpha=1.5), dict(temperature=math.nan)):
        with pytest.raises(PatconvError):
            distill.pp_distill(s, v, at, **kw)
    loss, stats = distill.pp_distill(s, v, at)
    for kw in (dict(dloss=loss[:3]), dict(dloss=loss.half()), dict(stats=stats[:, :4]), dict(stats=stats.t()), dict(out=s.half()), dict(out=s.t()), dict(out=s[:3])):
        with pytest.raises(ValueError):
            distill.pp_distill_backward(**({"dloss": loss, "logits": s, "stats": stats, "values": v, "indices": at} | kw))
    wide = torch.zeros(4, 104, device="cuda")
    with pytest.raises(PatconvError):
        distill.pp_distill_backward(loss, wide[:, :100], stats, v, at, out=wide.view(-1)[:400].view(4, 100))


def test_offsets_beyond_32_bits():
    """2.2e9 logits: the last rows' offsets pass 2^31.  They are compared with themselves alone."""
    rows, classes = 2304, 1 << 20
    if torch.cuda.mem_get_info()[0] < 30 << 30:
        pytest.skip("needs 30 GB of device memory")
    s = torch.empty((rows, classes), dtype=torch.float16, device="cuda")
    s[-3:].normal_()
    s[:-3].fill_(0.5)
    top = distill.pp_top_logits(s, 3, 2.0)
    alone = distill.pp_top_logits(s[-3:].clone(), 3, 2.0)
    assert torch.equal(top.indices[-3:], alone.indices) and torch.equal(top.values[-3:], alone.values)
    n = 2 * D.roundings(classes)                           # sums of other orders: a row alone has a cluster
    assert torch.allclose(top.rest[-3:], alone.rest, rtol=n) and top.indices[0].tolist() == [0, 1, 2]
    loss, stats = distill.pp_distill(s, *top, None, 2.0)
    loss1, stats1 = distill.pp_distill(s[-3:].clone(), *alone, None, 2.0)
    assert torch.allclose(loss[-3:], loss1, rtol=0, atol=100 * n) and torch.allclose(stats[-3:], stats1, rtol=n)
    g = torch.full((1,), 2.0 ** 15, device="cuda")
    want = distill.pp_distill_backward(g.expand(3), s[-3:].clone(), stats[-3:].clone(), *(t[-3:].clone() for t in top), None, 2.0)
    got = distill.pp_distill_backward(g.expand(rows), s, stats, *top, None, 2.0, out=s)
    assert torch.equal(got[-3:], want) and want.any()

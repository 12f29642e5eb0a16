"""The float64 oracle of distillation and block norm against differences and closed forms, and what the entry points refuse,
all on the CPU."""
import ctypes

import numpy as np
import pytest
import torch

from oracle import distill as D
from paper_2003_06513_gb300 import _lib, distill, norm

NULL, SHAPE, ALIGN, DTYPE, BUFFER, ARG = -1, -2, -6, -7, -9, -11


@pytest.fixture(scope="module")
def lib():
    return _lib.load()


# ------------------------------------------------------------------------------------- the oracle

def test_top_orders_ties_by_place_and_nan_first():
    s = np.array([[1.0, 3.0, -0.0, 3.0, 0.0, -np.inf], [np.nan, 2.0, np.inf, 2.0, 2.0, 1.0]])
    values, at, rest = D.top(s, 4, 2.0)
    assert at.tolist() == [[1, 3, 0, 2], [0, 2, 1, 3]]
    assert values[0].tolist() == [3, 3, 1, 0] and np.isnan(values[1, 0]) and values[1, 1] == np.inf
    assert rest[0] == pytest.approx(0.0) and rest[1] == pytest.approx(np.log(np.exp(1.0) + np.exp(0.5)))
    assert D.top(s[:, :4], 4, 1.0)[2][0] == -np.inf


def _problem(seed, rows=6, classes=9, k=3):
    rng = np.random.default_rng(seed)
    s, teacher = rng.standard_normal((2, rows, classes)) * 2
    values, at, rest = D.top(teacher, k, 1.5)
    return rng, s, teacher, values, at, rest


def test_without_a_rest_the_teacher_is_its_kept_classes():
    _, s, _, values, at, _ = _problem(1)
    loss = D.distill(s, values, at, None, None, 1.5, 1.0)[0]
    p = np.exp(values / 1.5) / np.exp(values / 1.5).sum(1, keepdims=True)
    q = np.exp(s / 1.5) / np.exp(s / 1.5).sum(1, keepdims=True)
    np.testing.assert_allclose(loss, 2.25 * (p * np.log(p / np.take_along_axis(q, at, 1))).sum(1))


def test_with_all_but_one_kept_the_rest_is_that_class():
    _, s, teacher, _, _, _ = _problem(2)
    values, at, rest = D.top(teacher, 8, 1.5)
    p = np.exp(teacher / 1.5) / np.exp(teacher / 1.5).sum(1, keepdims=True)
    q = np.exp(s / 1.5) / np.exp(s / 1.5).sum(1, keepdims=True)
    loss, _, grad = D.distill(s, values, at, rest, None, 1.5, 1.0)[:3]
    np.testing.assert_allclose(loss, 2.25 * (p * np.log(p / q)).sum(1))
    np.testing.assert_allclose(grad, 1.5 * (q - p))


@pytest.mark.parametrize("rest", [False, True])
@pytest.mark.parametrize("alpha", [0.0, 0.4, 1.0])
def test_the_gradient_is_that_of_differences(alpha, rest):
    rng, s, _, values, at, r = _problem(3)
    labels = np.array([0, 8, -1, 4, at[4, 0], 2])
    at[2] = -1                                          # nothing kept: with a rest alone there is nothing to learn
    at[3, 1] = at[3, 0]                                 # one class twice
    at[5, 2] = 9                                        # outside
    values[1, 2] = -np.inf
    r = r if rest else None
    grad = D.distill(s, values, at, r, labels, 1.5, alpha)[2]
    h = 1e-6
    for i in range(s.shape[0]):
        for v in range(s.shape[1]):
            up, down = s.copy(), s.copy()
            up[i, v] += h
            down[i, v] -= h
            d = (D.distill(up, values, at, r, labels, 1.5, alpha)[0] - D.distill(down, values, at, r, labels, 1.5, alpha)[0])[i] / (2 * h)
            assert abs(d - grad[i, v]) < 1e-7
    assert np.abs(grad.sum(1)).max() < 1e-12            # a shift of a row changes nothing
    if not rest:
        assert not grad[2].any()


@pytest.mark.parametrize("post", ["none", "rms", "layer"])
@pytest.mark.parametrize("pre,kind", [("none", "none"), ("rms", "silu"), ("layer", "relu"), ("layer", "none")])
def test_block_gradients_are_those_of_differences(post, pre, kind):
    rng = np.random.default_rng(4)
    shape, c, eps = (2, 5, 2, 3), 5, 1e-3
    x, b, dh, dy = rng.standard_normal((4,) + shape)
    par = {"pw": 1 + 0.3 * rng.standard_normal(c), "pb": rng.standard_normal(c), "scale": rng.standard_normal(c),
           "gate": rng.random((2, c)), "w": 1 + 0.3 * rng.standard_normal(c), "bias": rng.standard_normal(c)}
    if post == "none":
        par["pw"] = par["pb"] = None
    if pre == "none":
        par["w"] = par["bias"] = dy = None

    def value(x, b, par):
        h = D.block_h(x, b, post, par["pw"], par["pb"], par["scale"], par["gate"], eps)[0]
        y = D.block_y(h, pre, par["w"], par["bias"], kind, eps)[0]
        return (h * dh).sum() + (0 if dy is None else (y * dy).sum())

    h = D.block_h(x, b, post, par["pw"], par["pb"], par["scale"], par["gate"], eps)[0]
    got, _ = D.block_backward(dh, dy, h, b, post, par["pw"], par["pb"], par["scale"], par["gate"], pre, par["w"], par["bias"], kind, eps)
    names = {"dx": x, "dblock": b, "dpost_weight": par["pw"], "dpost_bias": par["pb"], "dscale": par["scale"], "dgate": par["gate"],
             "dweight": par["w"], "dbias": par["bias"]}
    for name, t in names.items():
        if t is None:
            continue
        for i in range(min(t.size, 12)):
            old = t.flat[i]
            t.flat[i] = old + 1e-6
            up = value(x, b, par)
            t.flat[i] = old - 1e-6
            down = value(x, b, par)
            t.flat[i] = old
            assert abs((up - down) / 2e-6 - got[name].flat[i]) < 2e-6, (name, i)


# ------------------------------------------------------------------------------------- refusals

def p(v):
    return ctypes.c_void_p(v) if v else None


def test_top_refusals(lib):
    def top(s=1 << 20, stride=100, dtype=0, rows=4, classes=100, k=5, t=1.0, values=256, indices=4096, rest=8192):
        return lib.pp_top_logits(p(s), stride, dtype, rows, classes, k, t, p(values), p(indices), p(rest), None)

    assert top(dtype=3) == DTYPE and top(k=0) == SHAPE and top(k=257, classes=1000, stride=1000) == SHAPE and top(k=101) == SHAPE
    assert top(rows=-1) == SHAPE and top(classes=0) == SHAPE and top(classes=(1 << 20) + 1, stride=1 << 21) == SHAPE and top(stride=99) == SHAPE
    for t in (0.0, -1.0, float("nan"), float("inf"), 1e-4, 1e4):
        assert top(t=t) == ARG
    for name in ("s", "values", "indices", "rest"):
        assert top(**{name: 0}) == NULL
    assert top(s=(1 << 20) + 2) == ALIGN and top(values=258) == ALIGN and top(indices=4097) == ALIGN and top(rest=8194) == ALIGN
    assert top(values=(1 << 20) + 16) == BUFFER and top(indices=256) == BUFFER and top(rest=4096) == BUFFER
    assert top(rows=0, s=0) == 0


def test_distill_refusals(lib):
    def fwd(s=1 << 20, stride=100, dtype=0, rows=4, classes=100, values=256, vt=0, indices=4096, kept=5, rest=8192, labels=12288, t=2.0,
            alpha=0.5, loss=16384, stats=20480):
        return lib.pp_distill(p(s), stride, dtype, rows, classes, p(values), vt, p(indices), kept, p(rest), p(labels), t, alpha, p(loss),
                              p(stats), None)

    assert fwd(dtype=3) == DTYPE and fwd(vt=-1) == DTYPE and fwd(kept=0) == SHAPE and fwd(kept=101) == SHAPE
    assert fwd(kept=257, classes=1000, stride=1000) == SHAPE and fwd(classes=0) == SHAPE and fwd(rows=-1) == SHAPE and fwd(stride=99) == SHAPE
    assert fwd(t=0.0) == ARG and fwd(t=float("nan")) == ARG and fwd(alpha=-0.1) == ARG and fwd(alpha=1.1) == ARG and fwd(alpha=float("nan")) == ARG
    for name in ("s", "values", "indices", "loss", "stats"):
        assert fwd(**{name: 0}) == NULL
    assert fwd(labels=12292) == ALIGN and fwd(rest=8193) == ALIGN and fwd(loss=16385) == ALIGN and fwd(stats=20482) == ALIGN
    assert fwd(loss=(1 << 20) + 64) == BUFFER and fwd(stats=16384) == BUFFER and fwd(loss=4096) == BUFFER and fwd(stats=12288) == BUFFER
    assert fwd(rows=0, s=0, loss=0) == 0

    def bwd(dloss=256, ds=0, s=1 << 20, stride=100, rows=4, classes=100, stats=512, values=1024, indices=2048, kept=5, rest=0, labels=0,
            out=1 << 22, t=1.0, alpha=0.5, dtype=0):
        return lib.pp_distill_backward(p(dloss), ds, p(s), stride, dtype, rows, classes, p(stats), p(values), 0, p(indices), kept, p(rest),
                                       p(labels), t, alpha, p(out), None)

    for name in ("dloss", "s", "stats", "values", "indices", "out"):
        assert bwd(**{name: 0}) == NULL
    assert bwd(ds=-1) == SHAPE and bwd(out=(1 << 22) + 2) == ALIGN and bwd(dloss=258) == ALIGN and bwd(dtype=7) == DTYPE
    assert bwd(out=(1 << 20) + 64) == BUFFER and bwd(out=1 << 20, stride=104) == BUFFER and bwd(out=512) == BUFFER
    assert bwd(rows=0, out=0) == 0


def test_block_refusals(lib):
    size = ctypes.c_size_t()
    assert lib.pp_block_norm_workspace_size(2, 4, 8, None) == NULL and lib.pp_block_norm_workspace_size(2, 4, 4097, ctypes.byref(size)) == SHAPE
    assert lib.pp_block_norm_workspace_size(2, 4, 8, ctypes.byref(size)) == 0 and size.value > 0
    ws = size.value
    assert lib.pp_block_norm_workspace_size(0, 4, 8, ctypes.byref(size)) == 0 and size.value == 0

    def fwd(x=1 << 20, px=8, sx=32, xt=0, b=1 << 21, pb=8, sb=32, dt=0, n=2, hw=4, c=8, post=1, pw=0, pbias=0, scale=0, gate=0, pre=1, w=0,
            bias=0, act=0, eps=1e-5, h=1 << 22, y=1 << 23):
        return lib.pp_block_norm(p(x), px, sx, xt, p(b), pb, sb, dt, n, hw, c, post, p(pw), p(pbias), p(scale), p(gate), pre, p(w), p(bias), act,
                                 eps, p(h), p(y), None)

    assert fwd(xt=1) == DTYPE and fwd(xt=1, dt=2) == DTYPE and fwd(dt=3) == DTYPE
    assert fwd(c=0) == SHAPE and fwd(c=4097) == SHAPE and fwd(n=-1) == SHAPE and fwd(px=7) == SHAPE and fwd(sb=-1) == SHAPE and fwd(n=1 << 20, hw=1 << 20) == SHAPE
    assert fwd(post=3) == ARG and fwd(pre=-1) == ARG and fwd(act=3) == ARG and fwd(eps=-1.0) == ARG and fwd(eps=float("inf")) == ARG
    assert fwd(pre=0, act=1) == ARG and fwd(pre=0, w=256) == ARG and fwd(post=0, pw=256) == ARG
    assert fwd(b=0) == ARG and fwd(b=0, post=0, gate=256) == ARG and fwd(b=0, post=0, pre=0) == ARG
    assert fwd(x=0) == NULL and fwd(h=0) == NULL and fwd(y=0) == NULL and fwd(b=0, post=0, y=0) == NULL
    assert fwd(x=(1 << 20) + 2) == ALIGN and fwd(pw=255) == ALIGN and fwd(gate=258) == ALIGN and fwd(h=(1 << 22) + 1) == ALIGN
    assert fwd(h=(1 << 20) + 64) == BUFFER and fwd(h=1 << 21) == BUFFER and fwd(y=1 << 20) == BUFFER and fwd(y=1 << 22) == BUFFER
    assert fwd(h=1 << 20, px=16, sx=64) == BUFFER and fwd(y=1 << 21, pb=16, sb=64) == BUFFER
    assert fwd(n=0, x=0) == 0 and fwd(hw=0, h=0, y=0) == 0

    def bwd(dh=1 << 18, dy=1 << 19, h=1 << 20, b=1 << 21, xt=0, dt=0, post=1, pre=1, pw=0, gate=0, dx=1 << 22, db=1 << 23, dpw=0, dgate=0, dw=0,
            space=1 << 24, wsb=ws, act=0):
        return lib.pp_block_norm_backward(p(dh), 8, 32, p(dy), 8, 32, p(h), 8, 32, xt, p(b), 8, 32, dt, 2, 4, 8, post, p(pw), None, None, p(gate),
                                          pre, None, None, act, 1e-5, p(dx), p(db), p(dpw), None, None, p(dgate), p(dw), None, p(space), wsb, None)

    assert bwd(dx=0) == NULL and bwd(db=0) == NULL and bwd(space=0) == NULL and bwd(h=0) == NULL
    assert bwd(wsb=ws - 1) == BUFFER and bwd(space=(1 << 24) + 8) == ALIGN and bwd(dx=(1 << 22) + 2) == ALIGN and bwd(dw=257) == ALIGN
    assert bwd(dgate=256) == ARG and bwd(post=0, dpw=256) == ARG and bwd(pre=0, dw=256, dy=0) == ARG and bwd(pre=0) == ARG
    assert bwd(b=0) == ARG and bwd(b=0, post=0, dpw=256) == ARG and bwd(xt=2, dt=1) == DTYPE
    assert bwd(dx=1 << 20) == BUFFER and bwd(dx=1 << 19) == BUFFER and bwd(db=1 << 21) == BUFFER and bwd(db=1 << 18) == BUFFER and bwd(db=1 << 22) == BUFFER


def test_sizes_and_strides_that_no_index_reaches(lib):
    """A CTA's last row, counted in 32 bits, and a tensor's last byte, in 64, have to exist."""
    size = ctypes.c_size_t()
    assert lib.pp_block_norm_workspace_size(1, (1 << 31) - (1 << 23), 1, ctypes.byref(size)) == SHAPE
    assert lib.pp_block_norm_workspace_size(3, (1 << 31) // 3 - (1 << 20), 1, ctypes.byref(size)) == SHAPE
    assert lib.pp_block_norm_workspace_size(1, (1 << 31) - (1 << 24) - 1, 1, ctypes.byref(size)) == 0
    big, out = p(1 << 20), p(1 << 40)
    assert lib.pp_block_norm(big, 8, 1 << 48, 0, big, 8, 32, 0, 8, 4, 8, 0, None, None, None, None, 0, None, None, 0, 1e-5, out, None, None) == SHAPE
    assert lib.pp_top_logits(big, 1 << 48, 0, 8, 100, 5, 1.0, out, p(1 << 41), p(1 << 42), None) == SHAPE
    assert lib.pp_top_logits(big, 100, 0, (1 << 27) + 1, 100, 5, 1.0, out, p(1 << 41), p(1 << 42), None) == SHAPE
    assert lib.pp_distill_backward(p(256), 1 << 48, big, 100, 0, 8, 100, p(1 << 41), p(1 << 42), 0, p(1 << 43), 5, None, None, 1.0, 0.5, out, None) == SHAPE


def test_bindings_refuse_what_is_not_on_the_gpu():
    s, at = torch.zeros(3, 10), torch.zeros(3, 2, dtype=torch.int32)
    for call in (lambda: distill.pp_top_logits(s, 2), lambda: distill.pp_distill(s, s[:, :2], at), lambda: distill.pp_distill_backward(s[:, 0], s, s, s, at),
                 lambda: distill.distill_loss(s, distill.TopLogits(s, at, None))):
        with pytest.raises(ValueError, match="CUDA"):
            call()
    x = torch.zeros(1, 8, 2, 2).contiguous(memory_format=torch.channels_last)
    for call in (lambda: norm.pp_block_norm(x, x), lambda: norm.pp_block_norm_backward(x, x, x, x), lambda: norm.block_norm(x, x)):
        with pytest.raises(ValueError, match="CUDA"):
            call()
    with pytest.raises(ValueError, match="pre must be"):
        norm.pp_block_norm(x, x, pre="batch")

"""Block norm on the GPU against the float64 oracle: shapes, types, kinds, strides, masks of parameters, extreme values,
streams.  Tolerances are the oracle's first-order bounds of fp32 error plus half a unit of the output type's last place."""
import numpy as np
import pytest
import torch

from oracle import distill as D
from paper_2003_06513_gb300 import norm
from paper_2003_06513_gb300._lib import PatconvError

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
ULP = {"f32": (2.0 ** -24, 0.0), "f16": (2.0 ** -11, 2.0 ** -25), "bf16": (2.0 ** -8, 0.0)}
NAMES = norm.BlockGrads._fields

# n, c, h, w: one value; one pixel; rows of less than a vector, of part of a warp, of a warp, of several; odd channels;
# samples that end inside a CTA's stretch, many small samples, one long one
SHAPES = [(1, 1, 1, 1), (3, 7, 1, 1), (2, 8, 3, 5), (1, 64, 32, 32), (5, 150, 21, 13), (2, 34, 9, 4), (3, 256, 7, 7), (2, 257, 5, 3), (4, 264, 6, 5),
          (2, 576, 7, 7), (1, 1023, 3, 5), (2, 960, 14, 14), (2, 2048, 3, 3), (1, 4096, 2, 5), (300, 12, 2, 2), (700, 24, 1, 1), (1, 16, 150, 211),
          (2, 96, 56, 56), (33, 128, 14, 14)]


def _image(a, dtype, wide=0, at=0):
    t = torch.from_numpy(np.ascontiguousarray(np.moveaxis(a, 1, 3))).to("cuda", DT[dtype])
    if wide:
        n, h, w, c = t.shape
        base = torch.full((n, h, w, c + wide), float("nan"), dtype=t.dtype, device="cuda")
        base[..., at:at + c] = t
        return base.permute(0, 3, 1, 2)[:, at:at + c]
    return t.permute(0, 3, 1, 2)


def _host(t):
    return t.detach().double().cpu().numpy()


def _held(rng, shape, dtype, spread=1.0, shift=0.3):
    """Values as the type holds them: every channel with its own spread and shift."""
    c = shape[1]
    x = rng.standard_normal(shape) * spread * (0.5 + rng.random((1, c, 1, 1))) + shift * rng.standard_normal((1, c, 1, 1))
    return torch.from_numpy(x).to(DT[dtype]).double().numpy()


def _parameters(rng, n, c, post, pre, given="all"):
    f = np.float32
    par = {"post_weight": (1 + 0.2 * rng.standard_normal(c)).astype(f), "post_bias": (0.2 * rng.standard_normal(c)).astype(f),
           "scale": (0.5 + 0.2 * rng.standard_normal(c)).astype(f), "gate": rng.random((n, c)).astype(f),
           "weight": (1 + 0.2 * rng.standard_normal(c)).astype(f), "bias": (0.2 * rng.standard_normal(c)).astype(f)}
    if post == "none":
        par["post_weight"] = par["post_bias"] = None
    if pre == "none":
        par["weight"] = par["bias"] = None
    if given != "all":
        par = {k: v if k in given else None for k, v in par.items()}
    return par


def _device(par):
    return {k: None if v is None else torch.from_numpy(v).cuda() for k, v in par.items()}


def _within(got, want, bound, dtype, what):
    rel, small = ULP[dtype]
    tol = bound + rel * (np.abs(want) + bound) + small + 2.0 ** -126
    worst = np.max(np.abs(got - want) / tol) if want.size else 0.0
    assert worst <= 1.0, f"{what}: {worst:.2f} times the tolerance"


def _check_forward(x, b, tx, tb, par, post, pre, act, stream, dtype, eps=1e-5):
    d = _device(par)
    h, y = norm.pp_block_norm(tx, tb, post, d["post_weight"], d["post_bias"], d["scale"], d["gate"], pre, d["weight"], d["bias"], act, eps)
    if b is not None:
        want, bound = D.block_h(x, b, post, par["post_weight"], par["post_bias"], par["scale"], par["gate"], eps)
        assert h.shape == tx.shape and h.dtype == tx.dtype and h.is_contiguous(memory_format=torch.channels_last)
        _within(_host(h), want, bound, stream, "h")
    else:
        assert h is tx
    if pre == "none":
        assert y is None
    else:
        want, bound = D.block_y(_host(h), pre, par["weight"], par["bias"], act, eps)
        assert y.dtype == (tx if tb is None else tb).dtype and y.is_contiguous(memory_format=torch.channels_last)
        _within(_host(y), want, bound, dtype, "y")
    return h, y


def _check_backward(dh, dy, h, b, tdh, tdy, th, tb, par, post, pre, act, stream, dtype, eps=1e-5):
    d = _device(par)
    got = norm.pp_block_norm_backward(tdh, tdy, th, tb, post, d["post_weight"], d["post_bias"], d["scale"], d["gate"], pre, d["weight"],
                                      d["bias"], act, eps)
    want, bound = D.block_backward(dh, dy, h, b, post, par["post_weight"], par["post_bias"], par["scale"], par["gate"], pre, par["weight"],
                                   par["bias"], act, eps)
    for name, t in got._asdict().items():
        there = name == "dx" or (b is not None if name == "dblock" else par[name[1:]] is not None)
        assert (t is not None) == there, name
        if t is None:
            continue
        if name not in want:                            # of y's norm, without a gradient of y
            assert not t.any()
            continue
        kind = stream if name == "dx" else dtype if name == "dblock" else "f32"
        assert t.dtype == DT[kind]
        _within(_host(t), want[name], bound[name], kind, name)
    return got


def _case(shape, dtype, stream, seed, post, pre, act, given="all"):
    rng = np.random.default_rng(seed)
    n, c, h, w = shape
    x, b = _held(rng, shape, stream, 1.5, 0.5), _held(rng, shape, dtype)
    par = _parameters(rng, n, c, post, pre, given)
    _check_forward(x, b, _image(x, stream), _image(b, dtype), par, post, pre, act, stream, dtype)
    dh, dy = _held(rng, shape, stream), _held(rng, shape, dtype) if pre != "none" else None
    _check_backward(dh, dy, x, b, _image(dh, stream), None if dy is None else _image(dy, dtype), _image(x, stream), _image(b, dtype), par, post, pre,
                    act, stream, dtype)


TYPES = [("f32", "f32"), ("f16", "f16"), ("bf16", "bf16"), ("f16", "f32"), ("bf16", "f32")]


@pytest.mark.parametrize("dtype,stream", TYPES)
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_shapes(shape, dtype, stream):
    k = shape[1] + shape[2]
    _case(shape, dtype, stream, k, ("rms", "layer")[k % 2], ("layer", "rms")[k // 2 % 2], ("none", "relu", "silu")[k % 3])


@pytest.mark.parametrize("act", ["none", "relu", "silu"])
@pytest.mark.parametrize("pre", ["none", "rms", "layer"])
@pytest.mark.parametrize("post", ["none", "rms", "layer"])
@pytest.mark.parametrize("shape", [(3, 48, 9, 11), (3, 320, 3, 5)], ids=str)
def test_kinds(shape, post, pre, act):
    if pre == "none" and act != "none":
        with pytest.raises(PatconvError):
            _case(shape, "f32", "f32", 1, post, pre, act)
        return
    _case(shape, "f32", "f32", 1, post, pre, act)


@pytest.mark.parametrize("given", [(), ("gate",), ("scale",), ("post_weight", "weight"), ("post_bias", "bias"), ("scale", "gate", "post_bias"), ("post_weight", "gate", "bias")], ids=str)
@pytest.mark.parametrize("shape", [(3, 40, 9, 11), (3, 320, 3, 5)], ids=str)
def test_missing_parameters(shape, given):
    _case(shape, "f32", "f32", 2, "layer", "rms", "silu", given)
    _case(shape, "f16", "f16", 3, "rms", "layer", "relu", given)


@pytest.mark.parametrize("dtype,stream", [("f32", "f32"), ("f16", "f16"), ("bf16", "f32")])
@pytest.mark.parametrize("wide,at", [(8, 8), (2, 2), (1, 0), (3, 1), (16, 4)])
@pytest.mark.parametrize("c", [24, 272])
def test_channels_of_a_wider_tensor(c, wide, at, dtype, stream):
    """Pixels further apart than C, at addresses of every alignment; what lies beside them is not read."""
    rng = np.random.default_rng(4)
    shape = (2, c, 5, 7)
    x, b, dh, dy = _held(rng, shape, stream), _held(rng, shape, dtype), _held(rng, shape, stream), _held(rng, shape, dtype)
    par = _parameters(rng, 2, c, "rms", "layer")
    for wx, wb in ((wide, 0), (0, wide), (wide, 8)):
        tx, tb = _image(x, stream, wx, at if wx == wide else 0), _image(b, dtype, wb, at if wb == wide else 0)
        _check_forward(x, b, tx, tb, par, "rms", "layer", "silu", stream, dtype)
        _check_backward(dh, dy, x, b, _image(dh, stream, wb, 0), _image(dy, dtype, wx, 0), tx, tb, par, "rms", "layer", "silu", stream, dtype)


def test_every_other_sample_and_one_sample_again():
    rng = np.random.default_rng(5)
    shape = (6, 40, 5, 6)
    x, b, dh, dy = (_held(rng, shape, "f32") for _ in range(4))
    par = _parameters(rng, 3, 40, "layer", "rms")
    tx, tb, td, ty = (_image(a, "f32") for a in (x, b, dh, dy))
    _check_forward(x[::2], b[1::2], tx[::2], tb[1::2], par, "layer", "rms", "relu", "f32", "f32")
    one, again = np.repeat(x[1:2], 3, 0), tx[1:2].expand(3, -1, -1, -1)
    _check_forward(one, b[:3], again, tb[:3], par, "layer", "rms", "none", "f32", "f32")
    _check_backward(dh[::2], np.repeat(dy[:1], 3, 0), one, b[3:], td[::2], ty[:1].expand(3, -1, -1, -1), again, tb[3:], par, "layer", "rms", "silu", "f32", "f32")


@pytest.mark.parametrize("shape", [(2, 48, 9, 11), (3, 320, 3, 5), (4, 1000, 1, 1)], ids=str)
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_the_norm_alone(shape, dtype):
    """Without a block: y = act(norm(x)), h is x itself; gradients of either or both."""
    rng = np.random.default_rng(6)
    x, dh, dy = (_held(rng, shape, dtype) for _ in range(3))
    par = _parameters(rng, shape[0], shape[1], "none", "layer", ("weight", "bias"))
    t = _image(x, dtype)
    _check_forward(x, None, t, None, par, "none", "layer", "relu", dtype, dtype)
    _check_backward(None, dy, x, None, None, _image(dy, dtype), t, None, par, "none", "layer", "relu", dtype, dtype)
    _check_backward(dh, dy, x, None, _image(dh, dtype), _image(dy, dtype), t, None, par, "none", "layer", "relu", dtype, dtype)


@pytest.mark.parametrize("shape", [(2, 48, 9, 11), (3, 320, 3, 5)], ids=str)
def test_one_gradient_alone(shape):
    rng = np.random.default_rng(7)
    x, b, dh, dy = (_held(rng, shape, "f32") for _ in range(4))
    par = _parameters(rng, shape[0], shape[1], "rms", "rms")
    t, tb = _image(x, "f32"), _image(b, "f32")
    _check_backward(dh, None, x, b, _image(dh, "f32"), None, t, tb, par, "rms", "rms", "silu", "f32", "f32")
    _check_backward(None, dy, x, b, None, _image(dy, "f32"), t, tb, par, "rms", "rms", "silu", "f32", "f32")


@pytest.mark.parametrize("c", [64, 150, 576])
@pytest.mark.parametrize("offset", [1e3, -3e4])
def test_values_far_from_zero(offset, c):
    """A layer norm of rows whose mean is thousands of spreads away; the oracle's bound has the mean's rounding in it."""
    rng = np.random.default_rng(8)
    shape = (2, c, 6, 7)
    x, b = (_held(rng, shape, "f32", shift=0.0) + offset for _ in range(2))
    x, b = (torch.from_numpy(a).float().double().numpy() for a in (x, b))
    dh, dy = _held(rng, shape, "f32"), _held(rng, shape, "f32")
    par = _parameters(rng, 2, c, "layer", "layer")
    _check_forward(x, b, _image(x, "f32"), _image(b, "f32"), par, "layer", "layer", "none", "f32", "f32")
    _check_backward(dh, dy, x, b, _image(dh, "f32"), _image(dy, "f32"), _image(x, "f32"), _image(b, "f32"), par, "layer", "layer", "none", "f32", "f32")


@pytest.mark.parametrize("c", [8, 12, 64, 150, 640])
@pytest.mark.parametrize("value", [0.0, 100.3, -7e8])
def test_constant_rows_give_the_bias(value, c):
    """A row of equal values has no spread: what fp32 leaves of it is below 2^-20 of the weight."""
    x = torch.full((2, c, 5, 3), value, device="cuda").contiguous(memory_format=torch.channels_last)
    w, bias = torch.full((c,), 1.7, device="cuda"), torch.linspace(-1, 1, c, device="cuda")
    _, y = norm.pp_block_norm(x, None, "none", pre="layer", weight=w, bias=bias)
    assert (y - bias.view(1, -1, 1, 1)).abs().max() <= 2.0 ** -20 * 1.7 * max(1.0, abs(value) * 2.0 ** -24 / 1e-5 ** 0.5)


def test_relu_sides_are_those_of_64_bits():
    """Values at the kink: fp32's z has the wrong sign for some of them, the gradient has not."""
    rng = np.random.default_rng(9)
    for c in (128, 512):
        shape = (2, c, 24, 24)
        x, dy = _held(rng, shape, "f32"), np.ones(shape)
        w = np.ones(c, np.float32)
        mean, root = x.mean(1, keepdims=True), np.sqrt(x.var(1, keepdims=True) + 1e-5)
        near = (-(x - mean) / root)[0, :, 3, 3].astype(np.float32)           # z of one pixel is a rounding from 0
        z = (x - mean) / root + near.reshape(1, -1, 1, 1).astype(np.float64)
        assert (np.abs(z[0, :, 3, 3]) < 1e-6).all()
        got = norm.pp_block_norm_backward(None, _image(dy, "f32"), _image(x, "f32"), None, "none", pre="layer", weight=torch.from_numpy(w).cuda(),
                                          bias=torch.from_numpy(near).cuda(), act="relu")
        # dbias counts the values above zero exactly
        np.testing.assert_array_equal(_host(got.dbias), (z > 0).sum((0, 2, 3)))


@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
@pytest.mark.parametrize("c", [24, 512])
def test_what_is_not_finite_stays_in_its_pixel(bad, c):
    rng = np.random.default_rng(10)
    shape = (2, c, 6, 5)
    tx, tb, td, ty = (_image(_held(rng, shape, "bf16"), "bf16") for _ in range(4))
    d = _device(_parameters(rng, 2, c, "layer", "rms"))
    args = ("layer", d["post_weight"], d["post_bias"], d["scale"], d["gate"], "rms", d["weight"], d["bias"], "silu")
    h, y = norm.pp_block_norm(tx, tb, *args)
    g = norm.pp_block_norm_backward(td, ty, h, tb, *args)
    spoilt = tb.clone(memory_format=torch.preserve_format)
    spoilt[1, 3, 2, 2] = bad
    h1, y1 = norm.pp_block_norm(tx, spoilt, *args)
    g1 = norm.pp_block_norm_backward(td, ty, h, spoilt, *args)
    keep = torch.ones_like(y, dtype=torch.bool)
    keep[1, :, 2, 2] = False
    assert torch.isnan(h1[1, :, 2, 2]).all() and torch.isnan(y1[1, :, 2, 2]).all() and torch.isnan(g1.dblock[1, :, 2, 2]).all()
    assert torch.equal(h1[keep], h[keep]) and torch.equal(y1[keep], y[keep]) and torch.equal(g1.dblock[keep], g.dblock[keep])
    assert torch.equal(g1.dx, g.dx) and torch.equal(g1.dgate[0], g.dgate[0])


@pytest.mark.parametrize("dtype", ["f32", "f16"])
@pytest.mark.parametrize("shape", [(2, 32, 20, 20), (1, 12, 1, 1), (3, 520, 4, 4), (1, 7, 5, 3)], ids=str)
def test_in_place(shape, dtype):
    rng = np.random.default_rng(11)
    tx, tb = (_image(_held(rng, shape, dtype), dtype) for _ in range(2))
    d = _device(_parameters(rng, shape[0], shape[1], "rms", "layer"))
    args = ("rms", d["post_weight"], d["post_bias"], d["scale"], d["gate"], "layer", d["weight"], d["bias"], "silu")
    want = norm.pp_block_norm(tx, tb, *args)
    versions = tx._version, tb._version
    h, y = norm.pp_block_norm(tx, tb, *args, out=(tx, tb))
    assert h.data_ptr() == tx.data_ptr() and y.data_ptr() == tb.data_ptr() and torch.equal(h, want[0]) and torch.equal(y, want[1])
    assert tx._version > versions[0] and tb._version > versions[1]


@pytest.mark.parametrize("dtype", ["f32", "f16"])
@pytest.mark.parametrize("shape", [(2, 32, 20, 20), (1, 12, 1, 1), (3, 520, 4, 4), (9, 256, 40, 40)], ids=str)
def test_gradients_in_place(shape, dtype):
    """dx over dh and dblock over dy, with rows read ahead of those that are written."""
    rng = np.random.default_rng(16)
    th, tb, td, ty = (_image(_held(rng, shape, dtype), dtype) for _ in range(4))
    d = _device(_parameters(rng, shape[0], shape[1], "layer", "rms"))
    args = ("layer", d["post_weight"], d["post_bias"], d["scale"], d["gate"], "rms", d["weight"], d["bias"], "silu")
    want = norm.pp_block_norm_backward(td, ty, th, tb, *args)
    versions = td._version, ty._version
    got = norm.pp_block_norm_backward(td, ty, th, tb, *args, out=(td, ty))
    assert got.dx.data_ptr() == td.data_ptr() and got.dblock.data_ptr() == ty.data_ptr()
    assert td._version > versions[0] and ty._version > versions[1] and all(torch.equal(a, b) for a, b in zip(got, want))
    with pytest.raises(PatconvError):
        norm.pp_block_norm_backward(td, ty, th, tb, *args, out=(th, None))


@pytest.mark.parametrize("c", [3, 24, 60, 150, 264])
@pytest.mark.parametrize("samples,pixels", [(1, 1), (1, 700), (2000, 1), (37, 50), (3, 5000)])
def test_samples_and_stretches(samples, pixels, c):
    """Gates' gradients of samples that begin, end and lie inside CTAs' stretches, and of more samples than there are CTAs."""
    _case((samples, c, pixels, 1), "f16", "f16", 17, "rms", "layer", "silu")


def test_nothing_to_do():
    for shape in ((0, 8, 3, 3), (2, 8, 0, 3)):
        x = torch.zeros(shape, device="cuda").contiguous(memory_format=torch.channels_last)
        one, gate = torch.ones(8, device="cuda"), torch.ones(shape[0], 8, device="cuda")
        h, y = norm.pp_block_norm(x, x, "rms", one, gate=gate, weight=one)
        assert h.shape == y.shape == x.shape
        g = norm.pp_block_norm_backward(x, x, h, x, "rms", one, gate=gate, weight=one)
        assert g.dx.shape == x.shape and not g.dweight.any() and not g.dpost_weight.any() and not g.dgate.any() and g.dgate.shape == gate.shape


@pytest.mark.parametrize("shape", [(1, 64, 32, 32), (5, 150, 21, 13), (3, 576, 14, 14)], ids=str)
def test_the_same_bits_again_on_another_stream_and_in_a_graph(shape):
    rng = np.random.default_rng(12)
    tx, tb, td, ty = (_image(_held(rng, shape, "f16"), "f16") for _ in range(4))
    d = _device(_parameters(rng, shape[0], shape[1], "rms", "layer"))
    args = ("rms", d["post_weight"], d["post_bias"], d["scale"], d["gate"], "layer", d["weight"], d["bias"], "relu")

    def both(**kw):
        h, y = norm.pp_block_norm(tx, tb, *args, **kw)
        return (h, y) + tuple(norm.pp_block_norm_backward(td, ty, h, tb, *args, **kw))

    want = both()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    again, other = both(), both(stream=side)
    torch.cuda.synchronize()
    graph, second = torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = both()
    with torch.cuda.graph(second):
        captured2 = both()
    for _ in range(3):
        graph.replay()
        second.replay()
    torch.cuda.synchronize()
    for a in (again, other, captured, captured2):
        assert all(torch.equal(x, z) for x, z in zip(want, a))


def test_caller_workspace_and_its_refusal():
    x = _image(_held(np.random.default_rng(13), (3, 48, 9, 7), "f32"), "f32")
    gate = torch.rand(3, 48, device="cuda")
    ws = torch.full((norm.block_workspace_bytes(x.shape),), 255, dtype=torch.uint8, device="cuda")
    a, b = (norm.pp_block_norm_backward(x, x, x, x, gate=gate, workspace=w) for w in (ws, None))
    assert torch.equal(a.dx, b.dx) and torch.equal(a.dgate, b.dgate)
    with pytest.raises(PatconvError):
        norm.pp_block_norm_backward(x, x, x, x, gate=gate, workspace=ws[:-16])


@pytest.mark.parametrize("wanted", ["both", "h", "y"])
def test_autograd(wanted):
    """block_norm's gradients are the formula's, for gradients in another order too, and where one output is not used."""
    rng = np.random.default_rng(14)
    shape = (2, 24, 6, 7)
    x, b, dh, dy = (_held(rng, shape, "f32") for _ in range(4))
    par = _parameters(rng, 2, 24, "layer", "rms")
    leaves = {"x": _image(x, "f32"), "block": _image(b, "f32")} | _device(par)
    leaves = {k: t.detach().clone(memory_format=torch.preserve_format).requires_grad_(True) for k, t in leaves.items()}
    h, y = norm.block_norm(leaves["x"], leaves["block"], "layer", leaves["post_weight"], leaves["post_bias"], leaves["scale"], leaves["gate"], "rms",
                           leaves["weight"], leaves["bias"], "silu")
    loss = 0
    if wanted != "y":
        loss = loss + (h.contiguous() * torch.from_numpy(dh).float().cuda()).sum()        # NCHW: the gradient comes in that order
    if wanted != "h":
        loss = loss + (y * torch.from_numpy(dy).float().cuda()).sum()
    loss.backward()
    want, bound = D.block_backward(dh if wanted != "y" else None, dy if wanted != "h" else None, _host(h), b, "layer", par["post_weight"], par["post_bias"],
                                   par["scale"], par["gate"], "rms", par["weight"], par["bias"], "silu", 1e-5)
    for name, leaf in leaves.items():
        name = "dx" if name == "x" else "d" + name
        if name in want:
            _within(_host(leaf.grad), want[name], bound[name], "f32", name)
        else:
            assert not leaf.grad.any()


def test_without_a_second_norm_in_autograd():
    rng = np.random.default_rng(18)
    x, b, dh = (_held(rng, (2, 24, 6, 7), "f32") for _ in range(3))
    tx, tb = (_image(a, "f32").detach().requires_grad_(True) for a in (x, b))
    h, y = norm.block_norm(tx, tb, "rms", pre="none")
    assert y is None
    (h * _image(dh, "f32")).sum().backward()
    want, bound = D.block_backward(dh, None, x, b, "rms", None, None, None, None, "none", None, None, "none", 1e-5)
    for leaf, name in ((tx, "dx"), (tb, "dblock")):
        _within(_host(leaf.grad), want[name], bound[name], "f32", name)


def test_a_captured_training_step():
    """Forward, loss and gradients of a block captured into a graph, replayed on other inputs."""
    rng = np.random.default_rng(19)
    shape = (2, 40, 8, 8)
    first, second = ([_image(_held(rng, shape, "f16"), "f16") for _ in range(2)] for _ in range(2))
    w = torch.rand(40, device="cuda")

    def step(x, b):
        x, b, leaf = (t.detach().requires_grad_(True) for t in (x, b, w))
        h, y = norm.block_norm(x, b, "layer", leaf, gate=torch.sigmoid(b.float().mean((2, 3))), pre="rms", act="silu")
        return torch.autograd.grad((h * y).float().sum(), (x, b, leaf))

    want = step(*second)
    static = [t.clone(memory_format=torch.preserve_format) for t in first]
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


def test_the_norm_alone_in_autograd():
    """Without a block h is x: what flows through both joins at the leaf."""
    rng = np.random.default_rng(15)
    x, dh, dy = (_held(rng, (2, 24, 6, 7), "f32") for _ in range(3))
    t = _image(x, "f32").detach().requires_grad_(True)
    h, y = norm.block_norm(t, None, "none", pre="layer")
    assert h is t
    (h * _image(dh, "f32") + y * _image(dy, "f32")).sum().backward()
    want, bound = D.block_backward(dh, dy, x, None, "none", None, None, None, None, "layer", None, None, "none", 1e-5)
    _within(_host(t.grad), want["dx"], bound["dx"] + 2 * D.U * np.abs(want["dx"]), "f32", "dx")


def test_refusals():
    nchw = torch.zeros(2, 8, 4, 4, device="cuda")
    x = nchw.contiguous(memory_format=torch.channels_last)
    one = torch.ones(8, device="cuda")
    for kw in (dict(x=nchw), dict(block=nchw), dict(block=x.half(), x=x.bfloat16()), dict(block=x[:1]), dict(block=x.cpu()), dict(x=x.half()),
               dict(post="batch"), dict(pre="group"), dict(act="gelu"), dict(weight=one[:4]), dict(bias=one.half()), dict(scale=one.cpu()), dict(gate=one),
               dict(gate=torch.ones(8, 2, device="cuda")), dict(out=(nchw, None)), dict(out=(None, x.half())), dict(x=x.double(), block=x.double())):
        with pytest.raises(ValueError):
            norm.pp_block_norm(**({"x": x, "block": x.clone(memory_format=torch.preserve_format)} | kw))
    for kw in (dict(eps=-1.0), dict(pre="none", act="relu"), dict(post="none", post_weight=one), dict(pre="none", weight=one), dict(block=None)):
        with pytest.raises(PatconvError):
            norm.pp_block_norm(**({"x": x, "block": x.clone(memory_format=torch.preserve_format)} | kw))
    for kw in (dict(dh=nchw), dict(dy=x.half()), dict(dh=x[:1]), dict(h=x.half()), dict(gate=one)):
        with pytest.raises(ValueError):
            norm.pp_block_norm_backward(**({"dh": x, "dy": x, "h": x, "block": x} | kw))
    with pytest.raises(PatconvError):
        norm.pp_block_norm_backward(x, x, x, x, pre="none")           # there is no y to have a gradient
    big = torch.zeros(1, 4104, 1, 1, device="cuda").contiguous(memory_format=torch.channels_last)
    with pytest.raises(PatconvError):
        norm.pp_block_norm(big, big)


def test_offsets_beyond_32_bits():
    """2.2e9 values: the last sample's offsets pass 2^31.  It is compared with itself alone."""
    n, c, h, w = 3, 64, 3400, 3400
    if torch.cuda.mem_get_info()[0] < 60 << 30:
        pytest.skip("needs 60 GB of device memory")
    x = torch.ones((n, h, w, c), dtype=torch.float16, device="cuda")
    x[2].normal_()
    t = x.permute(0, 3, 1, 2)
    gate = torch.rand(n, c, device="cuda")
    hh, y = norm.pp_block_norm(t, t, "layer", gate=gate, pre="layer", act="relu")
    h1, y1 = norm.pp_block_norm(t[2:], t[2:], "layer", gate=gate[2:], pre="layer", act="relu")
    assert torch.equal(hh[2:], h1) and torch.equal(y[2:], y1) and not y[:2].any() and torch.equal(hh[:2], t[:2])
    del y, y1
    g = norm.pp_block_norm_backward(t, t, hh, t, "layer", gate=gate, pre="layer", act="relu")
    g1 = norm.pp_block_norm_backward(t[2:], t[2:], h1, t[2:], "layer", gate=gate[2:], pre="layer", act="relu")
    assert torch.equal(g.dx[2:], g1.dx) and torch.equal(g.dblock[2:], g1.dblock)
    # sums over 1.2e7 pixels in another order
    assert torch.allclose(g.dgate[2], g1.dgate[0], rtol=1e-3, atol=1e-3 * float(g1.dgate.abs().max()))

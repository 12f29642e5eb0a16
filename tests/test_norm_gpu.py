"""Group norm with its activation on the GPU against the float64 oracle: shapes, types, strides, odd
sizes, extreme values, streams.  Tolerances are the oracle's first-order bounds of fp32 error plus half
a unit of the output type's last place."""
import numpy as np
import pytest
import torch

from oracle import train as T
from paper_2003_06513_gb300 import norm

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
# relative and absolute (subnormal) half units in the last place of the output types
ULP = {"f32": (2.0 ** -24, 0.0), "f16": (2.0 ** -11, 2.0 ** -25), "bf16": (2.0 ** -8, 0.0)}

# n, c, g, h, w: one value; one pixel; groups of one channel; odd channel counts and groups; rows that
# allow accesses of 16, 8, 4 and 2 bytes; several CTAs side by side, within groups and across; one group
SHAPES = [(1, 1, 1, 1, 1), (2, 6, 3, 1, 1), (2, 8, 8, 3, 5), (1, 64, 8, 32, 32), (3, 30, 10, 7, 9), (2, 150, 10, 45, 61),
          (4, 34, 17, 9, 4), (1, 1023, 1, 3, 5), (2, 2050, 2, 2, 3), (1, 4096, 32, 5, 7), (2, 520, 1, 6, 5), (32, 512, 32, 14, 14),
          (5, 8, 4, 56, 1), (2, 256, 32, 56, 56), (1, 64, 32, 224, 224), (3, 960, 32, 7, 7), (1, 4, 2, 1, 70000), (300, 12, 3, 2, 2)]


def _tensor(a, dtype, wide=0, at=0):
    """a [N, C, H, W] on the GPU in channels-last order, as channels at .. at + C of a tensor wider by
    ``wide`` channels."""
    t = torch.from_numpy(np.ascontiguousarray(np.moveaxis(a, 1, 3))).to("cuda", DT[dtype])
    if wide:
        n, h, w, c = t.shape
        base = torch.full((n, h, w, c + wide), float("nan"), dtype=t.dtype, device="cuda")
        base[..., at:at + c] = t
        return base.permute(0, 3, 1, 2)[:, at:at + c]
    return t.permute(0, 3, 1, 2)


def _host(t):
    return t.double().cpu().numpy()


def _inputs(shape, dtype, seed, offset=0.0):
    rng = np.random.default_rng(seed)
    c = shape[1]
    x = rng.standard_normal(shape) * (0.5 + rng.random((1, c, 1, 1))) + 0.3 * rng.standard_normal((1, c, 1, 1)) + offset
    x = torch.from_numpy(x).to(DT[dtype]).double().numpy()                  # as the type holds it
    ga = (1 + 0.2 * rng.standard_normal(c)).astype(np.float32)
    be = (0.2 * rng.standard_normal(c)).astype(np.float32)
    return x, ga, be


def _within(got, want, bound, dtype, what):
    rel, small = ULP[dtype]
    tol = bound + rel * (np.abs(want) + bound) + small
    worst = np.max(np.abs(got - want) / np.maximum(tol, 1e-300)) if want.size else 0.0
    assert worst <= 1.0, f"{what}: {worst:.2f} times the tolerance"


def _check_forward(x, t, g, ga, be, kind, dtype, eps=1e-5):
    dga, dbe = (torch.from_numpy(a).cuda() if a is not None else None for a in (ga, be))
    y, mean, rstd = norm.pp_group_norm(t, g, dga, dbe, eps, kind)
    want, wmean, wrstd, bound = T.norm_forward(x, g, ga, be, eps, kind)
    assert y.shape == t.shape and y.dtype == t.dtype and y.is_contiguous(memory_format=torch.channels_last)
    _within(_host(y), want, bound, dtype, "y")
    size = np.abs(x).reshape(x.shape[0], g, -1).mean(2)
    assert np.all(np.abs(_host(mean) - wmean) <= T.E * size)
    # the variance is off by twice the values' relative error, seen from the mean's size
    assert np.all(np.abs(_host(rstd) - wrstd) <= T.E * wrstd * (1 + size * wrstd))
    return y, mean, rstd


def _check_backward(x, dy, t, td, g, ga, be, kind, dtype):
    dga, dbe = (torch.from_numpy(a).cuda() if a is not None else None for a in (ga, be))
    _, mean, rstd, _ = T.norm_forward(x, g, ga, be, 1e-5, kind)
    mean, rstd = mean.astype(np.float32), rstd.astype(np.float32)
    got = norm.pp_group_norm_backward(td, t, torch.from_numpy(mean).cuda(), torch.from_numpy(rstd).cuda(), g, dga, dbe, kind)
    want, bounds = T.norm_backward(dy, x, mean, rstd, g, ga, be, kind)
    for a, b, e, what, dt in zip(got, want, bounds, ("dx", "dgamma", "dbeta"), (dtype, "f32", "f32")):
        _within(_host(a), b, e, dt, what)
    return got


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_forward(shape, dtype):
    n, c, g, h, w = shape
    x, ga, be = _inputs((n, c, h, w), dtype, c + h)
    kind = ("none", "relu", "silu")[(c + h) % 3]
    _check_forward(x, _tensor(x, dtype), g, ga, be, kind, dtype)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_backward(shape, dtype):
    n, c, g, h, w = shape
    x, ga, be = _inputs((n, c, h, w), dtype, c + h + 1)
    dy, _, _ = _inputs((n, c, h, w), dtype, c + h + 2)
    kind = ("none", "relu", "silu")[(c + h + 1) % 3]
    _check_backward(x, dy, _tensor(x, dtype), _tensor(dy, dtype), g, ga, be, kind, dtype)


@pytest.mark.parametrize("kind", ["none", "relu", "silu"])
@pytest.mark.parametrize("affine", ["both", "gamma", "beta", "neither"])
def test_activations_and_missing_parameters(kind, affine):
    x, ga, be = _inputs((2, 48, 9, 11), "f32", 5)
    dy, _, _ = _inputs((2, 48, 9, 11), "f32", 6)
    ga, be = ga if affine in ("both", "gamma") else None, be if affine in ("both", "beta") else None
    _check_forward(x, _tensor(x, "f32"), 6, ga, be, kind, "f32")
    _check_backward(x, dy, _tensor(x, "f32"), _tensor(dy, "f32"), 6, ga, be, kind, "f32")


@pytest.mark.parametrize("dtype", ["f32", "f16"])
@pytest.mark.parametrize("wide,at", [(8, 8), (2, 2), (1, 0), (3, 1)])
def test_channels_of_a_wider_tensor(wide, at, dtype):
    """Pixels further apart than C, at addresses of every alignment; what lies beside them is not read."""
    x, ga, be = _inputs((2, 24, 13, 17), dtype, 7)
    dy, _, _ = _inputs((2, 24, 13, 17), dtype, 8)
    _check_forward(x, _tensor(x, dtype, wide, at), 4, ga, be, "silu", dtype)
    _check_backward(x, dy, _tensor(x, dtype, wide, at), _tensor(dy, dtype, 4, 4), 4, ga, be, "silu", dtype)
    _check_backward(x, dy, _tensor(x, dtype), _tensor(dy, dtype, wide, at), 4, ga, be, "relu", dtype)


def test_every_other_sample_and_one_sample_again():
    x, ga, be = _inputs((6, 16, 5, 6), "f32", 9)
    t = _tensor(x, "f32")
    _check_forward(x[::2], t[::2], 4, ga, be, "relu", "f32")
    _check_forward(np.repeat(x[1:2], 3, 0), t[1:2].expand(3, -1, -1, -1), 4, ga, be, "relu", "f32")


@pytest.mark.parametrize("offset", [1e3, -3e4])
def test_values_far_from_zero(offset):
    """The variance of values whose mean is thousands of spreads away."""
    x, ga, be = _inputs((2, 32, 40, 40), "f32", 10, offset)
    _check_forward(x, _tensor(x, "f32"), 8, ga, be, "none", "f32")


def test_one_outlier():
    """A group whose first value lies far from the others: its squares are not taken from there."""
    x, ga, be = _inputs((1, 8, 30, 30), "f32", 11)
    x[0, 0, 0, 0] = 3e4
    _check_forward(x, _tensor(x, "f32"), 2, ga, be, "none", "f32")


@pytest.mark.parametrize("value", [0.0, 100.3, -7e8])
def test_constant_groups_give_beta_exactly(value):
    ga, be = torch.full((12,), 1.7, device="cuda"), torch.linspace(-1, 1, 12, device="cuda")
    x = torch.full((2, 12, 21, 19), value, device="cuda").contiguous(memory_format=torch.channels_last)
    y, mean, rstd = norm.pp_group_norm(x, 3, ga, be)
    assert torch.equal(y, be.view(1, -1, 1, 1).expand_as(y)) and torch.equal(mean, x[:, :3, 0, 0])
    assert torch.allclose(rstd, torch.full_like(rstd, 1e-5 ** -0.5), rtol=1e-6)


def test_a_group_of_one_value_has_no_gradient():
    x, ga, be = _inputs((3, 8, 1, 1), "f32", 12)
    t, td = _tensor(x, "f32"), _tensor(x[::-1], "f32")
    _, mean, rstd = norm.pp_group_norm(t, 8)
    dx, dgamma, _ = norm.pp_group_norm_backward(td, t, mean, rstd, 8, torch.from_numpy(ga).cuda(), torch.from_numpy(be).cuda())
    assert not dx.any() and not dgamma.any()


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_what_is_not_finite_stays_in_its_group(bad, dtype):
    x, ga, be = _inputs((2, 24, 9, 10), dtype, 13)
    t = _tensor(x, dtype)
    dga, dbe = torch.from_numpy(ga).cuda(), torch.from_numpy(be).cuda()
    clean, cm, cr = norm.pp_group_norm(t, 4, dga, dbe, act="relu")
    spoilt = t.clone(memory_format=torch.preserve_format)
    spoilt[1, 8, 4, 4] = bad
    y, mean, rstd = norm.pp_group_norm(spoilt, 4, dga, dbe, act="relu")
    assert torch.isnan(y[1, 6:12]).all()
    keep = torch.ones_like(y, dtype=torch.bool)
    keep[1, 6:12] = False
    assert torch.equal(y[keep], clean[keep])
    assert torch.isfinite(mean).sum() == 7 and torch.equal(rstd[0], cr[0])
    dy = torch.ones_like(t)
    dx, dgamma, dbeta = norm.pp_group_norm_backward(dy, spoilt, mean, rstd, 4, dga, dbe, "relu")
    assert torch.isnan(dx[1, 6:12]).all() and torch.isfinite(dx[keep]).all()
    assert torch.isnan(dgamma[6:12]).all() and torch.isfinite(dgamma[:6]).all() and torch.isfinite(dgamma[12:]).all()


def test_large_negative_silu_is_zero_and_not_nan():
    x = torch.tensor([[-1.0], [1.0]], device="cuda").view(1, 2, 1, 1).contiguous(memory_format=torch.channels_last)
    y, mean, rstd = norm.pp_group_norm(x, 1, torch.full((2,), 1e4, device="cuda"), None, 0.0, "silu")
    assert abs(float(y[0, 0])) < 1e-30 and float(y[0, 1]) == pytest.approx(1e4, rel=1e-5)
    dx, dg, _ = norm.pp_group_norm_backward(torch.ones_like(x), x, mean, rstd, 1, torch.full((2,), 1e4, device="cuda"), None, "silu")
    assert torch.isfinite(dx).all() and torch.isfinite(dg).all()


def test_in_place():
    x, ga, be = _inputs((2, 32, 20, 20), "f16", 14)
    t, dga, dbe = _tensor(x, "f16"), torch.from_numpy(ga).cuda(), torch.from_numpy(be).cuda()
    want, mean, rstd = norm.pp_group_norm(t, 8, dga, dbe, act="silu")
    dy = torch.randn_like(t)
    dwant = norm.pp_group_norm_backward(dy, t, mean, rstd, 8, dga, dbe, "silu")
    dgot = norm.pp_group_norm_backward(dy, t, mean, rstd, 8, dga, dbe, "silu", out=dy)
    assert dgot[0].data_ptr() == dy.data_ptr() and all(torch.equal(a, b) for a, b in zip(dgot, dwant))
    got, _, _ = norm.pp_group_norm(t, 8, dga, dbe, act="silu", out=t)
    assert got.data_ptr() == t.data_ptr() and torch.equal(got, want)


def test_nothing_to_do():
    for shape in ((0, 8, 3, 3), (2, 8, 0, 3)):
        x = torch.zeros(shape, device="cuda").contiguous(memory_format=torch.channels_last)
        y, mean, rstd = norm.pp_group_norm(x, 2)
        assert y.shape == x.shape
        dx, dg, db = norm.pp_group_norm_backward(x, x, mean, rstd, 2)
        assert dx.shape == x.shape and not dg.any() and not db.any()


@pytest.mark.parametrize("shape", [(1, 64, 8, 32, 32), (4, 64, 32, 112, 112), (2, 150, 10, 45, 61)], ids=str)
def test_the_same_bits_again_on_another_stream_and_in_a_graph(shape):
    n, c, g, h, w = shape
    x, ga, be = _inputs((n, c, h, w), "f32", 15)
    dy, _, _ = _inputs((n, c, h, w), "f32", 16)
    t, td, dga, dbe = _tensor(x, "f32"), _tensor(dy, "f32"), torch.from_numpy(ga).cuda(), torch.from_numpy(be).cuda()

    def both(**kw):
        y, mean, rstd = norm.pp_group_norm(t, g, dga, dbe, act="silu", **kw)
        return (y, mean, rstd) + norm.pp_group_norm_backward(td, t, mean, rstd, g, dga, dbe, "silu", **kw)

    want = both()
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    again, other = both(), both(stream=s)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = both()
    for _ in range(3):
        graph.replay()
    torch.cuda.synchronize()
    for a, b, e, f in zip(want, again, other, captured):
        assert torch.equal(a, b) and torch.equal(a, e) and torch.equal(a, f)


def test_caller_workspace_and_its_refusal():
    x, ga, be = _inputs((2, 64, 40, 40), "f32", 17)
    t = _tensor(x, "f32")
    ws = torch.full((norm.workspace_bytes(t.shape, 8),), 255, dtype=torch.uint8, device="cuda")
    assert torch.equal(norm.pp_group_norm(t, 8, workspace=ws)[0], norm.pp_group_norm(t, 8)[0])
    if ws.numel():
        with pytest.raises(norm._lib.PatconvError):
            norm.pp_group_norm(t, 8, workspace=ws[:-16])


def test_autograd_against_the_formula():
    """group_norm's gradients are pp_group_norm_backward's, for a gradient in another order too."""
    x, ga, be = _inputs((2, 16, 6, 7), "f32", 18)
    t = _tensor(x, "f32").detach().requires_grad_(True)
    dga, dbe = (torch.from_numpy(a).cuda().requires_grad_(True) for a in (ga, be))
    weight = torch.randn(2, 16, 6, 7, device="cuda")                         # NCHW: dy comes in that order
    y = norm.group_norm(t, 4, dga, dbe, act="silu")
    (y.contiguous() * weight).sum().backward()
    want, bounds = T.norm_backward(_host(weight), x, *T.norm_forward(x, 4, ga, be, 1e-5, "silu")[1:3], 4, ga, be, "silu")
    for got, w, e in zip((t.grad, dga.grad, dbe.grad), want, bounds):
        # mean and rstd are the kernel's: twice the bound for their roundings, and of the largest for cancellation
        assert np.all(np.abs(_host(got) - w) <= 2 * e + T.E * np.abs(w).max())
    y = norm.group_norm(t, 4, dga, None)
    y.sum().backward()
    with torch.no_grad():
        assert norm.group_norm(t, 4).requires_grad is False


def test_refusals():
    x = torch.zeros(2, 8, 4, 4, device="cuda")
    with pytest.raises(ValueError, match="channels last"):
        norm.pp_group_norm(x, 2)
    x = x.contiguous(memory_format=torch.channels_last)
    one = torch.ones(8, device="cuda")
    for kw in (dict(groups=3), dict(groups=0), dict(groups=2, act="gelu"), dict(groups=2, weight=one[:4]),
               dict(groups=2, weight=one.half()), dict(groups=2, bias=one.cpu()), dict(groups=2, out=torch.zeros(2, 8, 4, 4, device="cuda")),
               dict(groups=2, out=x.half())):
        with pytest.raises(ValueError):
            norm.pp_group_norm(x, **kw)
    with pytest.raises(ValueError):
        norm.pp_group_norm(x.double(), 2)
    _, mean, rstd = norm.pp_group_norm(x, 2)
    for kw in (dict(dy=x.half()), dict(dy=x[:1]), dict(mean=mean[:1]), dict(rstd=rstd.double()), dict(dy=torch.zeros(2, 8, 4, 4, device="cuda"))):
        args = dict(dy=x, x=x, mean=mean, rstd=rstd, groups=2) | kw
        with pytest.raises(ValueError):
            norm.pp_group_norm_backward(**args)
    with pytest.raises(norm._lib.PatconvError):
        norm.pp_group_norm(x, 2, eps=-1.0)


def test_offsets_beyond_32_bits():
    """3.2e9 elements: the last sample's offsets pass 2^31.  It is compared with itself alone."""
    n, c, h, w = 3, 64, 4100, 4100
    if torch.cuda.mem_get_info()[0] < 40 << 30:
        pytest.skip("needs 40 GB of device memory")
    x = torch.empty((n, h, w, c), dtype=torch.float16, device="cuda")
    x[2].normal_()
    x[:2].fill_(1.0)
    t = x.permute(0, 3, 1, 2)
    y, mean, rstd = norm.pp_group_norm(t, 32, act="relu")
    alone, m1, r1 = norm.pp_group_norm(t[2:], 32, act="relu")
    assert torch.allclose(mean[2:], m1, rtol=0, atol=1e-6) and torch.allclose(rstd[2:], r1, rtol=1e-6)
    part = x[2].view(-1, 32, 2)[:1 << 20].double()
    want = ((part - mean[2, :, None].double()) * rstd[2, :, None].double()).clamp_min(0).view(-1, c)
    got = y[2].permute(1, 2, 0).reshape(-1, c)
    assert torch.allclose(got[:1 << 20].double(), want, rtol=2.0 ** -10, atol=1e-5)
    assert torch.allclose(got[-4096:].float(), alone[0].permute(1, 2, 0).reshape(-1, c)[-4096:].float(), rtol=2.0 ** -9, atol=1e-5)
    assert not y[:2].any()
    dx, _, _ = norm.pp_group_norm_backward(y, t, mean, rstd, 32, act="relu", out=y)
    assert torch.isfinite(dx[2]).all() and not dx[:2].any() and dx[2, :, -1].any()


@pytest.mark.parametrize("dtype,size", [("f32", 1e13), ("f32", 1e15), ("f32", 1e16), ("f32", 1e-14), ("f32", 1e-16),
                                        ("bf16", 1e15), ("bf16", 1e-14)])
@pytest.mark.parametrize("shape", [(2, 32, 4, 9, 11), (1, 8192, 1, 2, 2)], ids=str)
def test_gradients_of_values_of_any_size(shape, dtype, size):
    """Spreads whose rstd^3 fp32 does not hold, without an eps beside them; resident and streamed."""
    n, c, g, h, w = shape
    assert norm.plan((n, c, h, w), g, DT[dtype], True)["path"] == (1 if c == 8192 else 2)
    x, ga, be = _inputs((n, c, h, w), dtype, 22)
    x = torch.from_numpy(x * size).to(DT[dtype]).double().numpy()
    dy, _, _ = _inputs((n, c, h, w), dtype, 23)
    _, mean, rstd, _ = T.norm_forward(x, g, ga, be, 0.0, "silu")
    mean, rstd = mean.astype(np.float32), rstd.astype(np.float32)
    got = norm.pp_group_norm_backward(_tensor(dy, dtype), _tensor(x, dtype), torch.from_numpy(mean).cuda(), torch.from_numpy(rstd).cuda(), g,
                                      torch.from_numpy(ga).cuda(), torch.from_numpy(be).cuda(), "silu")
    want, bounds = T.norm_backward(dy, x, mean, rstd, g, ga, be, "silu")
    for a, b, e, what, dt in zip(got, want, bounds, ("dx", "dgamma", "dbeta"), (dtype, "f32", "f32")):
        _within(_host(a), b, e, dt, what)
    # the forward pass of the same values, whose squares fp32 holds
    _check_forward(x, _tensor(x, dtype), g, ga, be, "silu", dtype, 0.0)


@pytest.mark.parametrize("dtype", ["f32", "f16"])
@pytest.mark.parametrize("shape", [(1, 64, 8, 32, 32), (1, 12, 4, 1, 1), (3, 12, 4, 1, 1), (1, 8192, 1, 2, 2), (1, 1, 1, 5, 3)], ids=str)
def test_in_place_of_one_sample_and_of_one_pixel(shape, dtype):
    """Where there is one sample or one pixel the strides between them say nothing."""
    n, c, g, h, w = shape
    x, ga, be = _inputs((n, c, h, w), dtype, 21)
    t, dga, dbe = _tensor(x, dtype), torch.from_numpy(ga).cuda(), torch.from_numpy(be).cuda()
    want, mean, rstd = norm.pp_group_norm(t, g, dga, dbe, act="silu")
    dy = torch.randn_like(t)
    dwant = norm.pp_group_norm_backward(dy, t, mean, rstd, g, dga, dbe, "silu")
    dgot = norm.pp_group_norm_backward(dy, t, mean, rstd, g, dga, dbe, "silu", out=dy)
    assert dgot[0].data_ptr() == dy.data_ptr() and all(torch.equal(a, b) for a, b in zip(dgot, dwant))
    got, _, _ = norm.pp_group_norm(t, g, dga, dbe, act="silu", out=t)
    assert got.data_ptr() == t.data_ptr() and torch.equal(got, want)


def test_moments_of_no_pixels_are_nan():
    x = torch.zeros((2, 8, 0, 3), device="cuda").contiguous(memory_format=torch.channels_last)
    for value in (1.0, -2.0):
        junk = [torch.full((2, 2), value, device="cuda") for _ in range(8)]
        del junk                                          # memory that the outputs are likely to take
        y, mean, rstd = norm.pp_group_norm(x, 2)
        assert y.shape == x.shape and torch.isnan(mean).all() and torch.isnan(rstd).all()
    _, mean, rstd = norm.pp_group_norm(torch.zeros((0, 8, 4, 3), device="cuda").contiguous(memory_format=torch.channels_last), 2)
    assert mean.shape == rstd.shape == (0, 2)

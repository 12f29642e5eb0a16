"""Block norm on the GPU where a value is not finite: what the formula has in 64 bits, NaN for NaN, in every kind of norm."""
import numpy as np
import pytest
import torch

from oracle import distill as D
from paper_2003_06513_gb300 import norm

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
ULP = {"f32": (2.0 ** -24, 2.0 ** -126), "f16": (2.0 ** -11, 2.0 ** -25), "bf16": (2.0 ** -8, 2.0 ** -126)}
BAD = {"nan": np.nan, "inf": np.inf, "-inf": -np.inf}


def _held(rng, shape, dtype):
    x = rng.standard_normal(shape) * (0.5 + rng.random((1, shape[1], 1, 1))) + 0.3 * rng.standard_normal((1, shape[1], 1, 1))
    return torch.from_numpy(x).to(DT[dtype]).double().numpy()


def _image(a, dtype):
    return torch.from_numpy(np.ascontiguousarray(np.moveaxis(a, 1, 3))).to("cuda", DT[dtype]).permute(0, 3, 1, 2)


def _host(t):
    return t.detach().double().cpu().numpy()


def _same(got, want, bound, dtype, what):
    """What is not finite is so on both sides, of the same sign; the rest agrees to the oracle's bound and half a unit in the last place."""
    fine = np.isfinite(want)
    np.testing.assert_array_equal(got[~fine], want[~fine], err_msg=what)
    rel, small = ULP[dtype]
    tol = bound[fine] + rel * (np.abs(want[fine]) + bound[fine]) + small
    worst = np.max(np.abs(got[fine] - want[fine]) / tol) if fine.any() else 0.0
    assert worst <= 1.0, f"{what}: {worst:.2f} times the tolerance"


def _parameters(rng, n, c, post, pre):
    f = np.float32
    par = {"post_weight": 1 + 0.2 * rng.standard_normal(c), "post_bias": 0.2 * rng.standard_normal(c), "scale": 0.4 + 0.2 * rng.random(c),
           "gate": 0.1 + rng.random((n, c)), "weight": 1 + 0.2 * rng.standard_normal(c), "bias": 0.2 * rng.standard_normal(c)}
    missing = (("post_weight", "post_bias") if post == "none" else ()) + (("weight", "bias") if pre == "none" else ())
    return {k: None if k in missing else v.astype(f) for k, v in par.items()}


def _check(shape, dtype, stream, post, pre, act, x, b, h, dh, dy, par):
    d = {k: None if v is None else torch.from_numpy(v).cuda() for k, v in par.items()}
    args = (post, d["post_weight"], d["post_bias"], d["scale"], d["gate"], pre, d["weight"], d["bias"], act)
    with np.errstate(all="ignore"):
        got_h, got_y = norm.pp_block_norm(_image(x, stream), _image(b, dtype), *args)
        want, bound = D.block_h(x, b, post, par["post_weight"], par["post_bias"], par["scale"], par["gate"], 1e-5)
        _same(_host(got_h), want, bound, stream, "h")
        if pre != "none":
            want, bound = D.block_y(_host(got_h), pre, par["weight"], par["bias"], act, 1e-5)
            _same(_host(got_y), want, bound, dtype, "y")
        g = norm.pp_block_norm_backward(_image(dh, stream), None if pre == "none" else _image(dy, dtype), _image(h, stream), _image(b, dtype), *args)
        want, bound = D.block_backward(dh, None if pre == "none" else dy, h, b, post, par["post_weight"], par["post_bias"], par["scale"], par["gate"],
                                       pre, par["weight"], par["bias"], act, 1e-5)
        for name, t in g._asdict().items():
            if t is not None:
                _same(_host(t), want[name], bound[name], stream if name == "dx" else dtype if name == "dblock" else "f32", name)


@pytest.mark.parametrize("bad", list(BAD))
@pytest.mark.parametrize("post,pre", [("rms", "rms"), ("layer", "layer"), ("none", "rms"), ("rms", "layer"), ("layer", "rms"), ("none", "layer"), ("rms", "none")])
@pytest.mark.parametrize("c", [8, 24, 150, 256, 512])
def test_a_value_that_is_not_finite(c, post, pre, bad):
    """One channel of a pixel, the row's first and the row's last: of the block's output, of the stream before it, and in the backward
    pass of the stream after it."""
    dtype, stream = {8: ("f32", "f32"), 24: ("f16", "f16"), 150: ("bf16", "f32"), 256: ("bf16", "bf16"), 512: ("f16", "f16")}[c]
    rng = np.random.default_rng(c)
    shape = (2, c, 5, 4)
    x, h, dh = (_held(rng, shape, stream) for _ in range(3))
    b, dy = (_held(rng, shape, dtype) for _ in range(2))
    par = _parameters(rng, 2, c, post, pre)
    for act in ("none",) if pre == "none" else ("relu", "silu"):
        for channel in (0, c - 1):
            for where in ("block", "stream"):
                spoilt = [a.copy() for a in (x, b, h)]
                for a in spoilt[1:2] if where == "block" else spoilt[::2]:
                    a[1, channel, 2, 1] = BAD[bad]
                _check(shape, dtype, stream, post, pre, act, *spoilt, dh, dy, par)


def test_rows_up_to_the_limit():
    """2.13e9 pixels of one channel in two samples with a gate: the second one's rows plus its pixels pass 2^31.  Compared with itself alone;
    its sums, of some 27 thousand positive terms a thread, are off by as many roundings at most on either side."""
    n, h, w = 2, 35500, 30000
    if torch.cuda.mem_get_info()[0] < 60 << 30:
        pytest.skip("needs 60 GB of device memory")
    assert n * h * w < 2 ** 31 - 2 ** 24 < n * h * w + h * w

    def values(seed):
        t = torch.empty((n, h, w, 1), dtype=torch.float16, device="cuda")
        return t.uniform_(0.5, 2.0, generator=torch.Generator("cuda").manual_seed(seed)).permute(0, 3, 1, 2)

    x, b, dh, dy = (values(seed) for seed in range(4))
    gate, scale = torch.tensor([[0.7], [0.4]], device="cuda"), torch.ones(1, device="cuda")
    kinds = {"post": "rms", "pre": "rms", "scale": scale, "act": "relu"}
    out_h, y = norm.pp_block_norm(x, b, gate=gate, **kinds)
    h1, y1 = norm.pp_block_norm(x[1:], b[1:], gate=gate[1:], **kinds)
    assert torch.equal(out_h[1:], h1) and torch.equal(y[1:], y1)
    del y, y1, x
    g = norm.pp_block_norm_backward(dh, dy, out_h, b, gate=gate, **kinds)
    g1 = norm.pp_block_norm_backward(dh[1:], dy[1:], h1, b[1:], gate=gate[1:], **kinds)
    assert torch.equal(g.dx[1:], g1.dx) and torch.equal(g.dblock[1:], g1.dblock)
    assert abs(float(g.dgate[1]) - float(g1.dgate[0])) <= 2 * 27000 * 2.0 ** -24 * float(g1.dgate[0])

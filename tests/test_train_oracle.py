"""The oracle of the retraining operators against differences, torch's CPU operations and itself, and
the refusals of their C entry points and Python bindings (no GPU)."""
import ctypes
import math

import numpy as np
import pytest
import torch

from oracle import train as T
from paper_2003_06513_gb300 import _lib, norm, optim

NULL, SHAPE, ALIGN, DTYPE, NOT_BOUND, BUFFER, ARG = -1, -2, -6, -7, -8, -9, -11


# ------------------------------------------------------------------------------------ the oracle

@pytest.mark.parametrize("kind", ["none", "relu", "silu"])
@pytest.mark.parametrize("shape,groups", [((2, 6, 3, 4), 3), ((1, 5, 1, 2), 1), ((3, 4, 2, 2), 4)])
def test_norm_forward_is_torchs(kind, shape, groups):
    rng = np.random.default_rng(0)
    x, ga, be = rng.standard_normal(shape) + 0.5, rng.standard_normal(shape[1]), rng.standard_normal(shape[1])
    y, mean, rstd, _ = T.norm_forward(x, groups, ga, be, 1e-5, kind)
    t = torch.nn.functional.group_norm(torch.from_numpy(x), groups, torch.from_numpy(ga), torch.from_numpy(be), 1e-5)
    t = {"none": t, "relu": t.relu(), "silu": torch.nn.functional.silu(t)}[kind]
    np.testing.assert_allclose(y, t.numpy(), rtol=1e-12, atol=1e-12)
    assert mean.shape == rstd.shape == (shape[0], groups)


@pytest.mark.parametrize("kind", ["none", "relu", "silu"])
def test_norm_backward_against_differences(kind):
    """Central differences of sum(y w) in 64 bits: truncation h^2 and cancellation 1e-16 / h at h = 1e-5."""
    rng = np.random.default_rng(1)
    shape, groups, eps, h = (2, 6, 3, 2), 2, 1e-5, 1e-5
    x, w = rng.standard_normal(shape), rng.standard_normal(shape)
    ga, be = 1 + 0.3 * rng.standard_normal(6), 0.3 * rng.standard_normal(6)

    def loss(x, ga, be):
        return float((T.norm_forward(x, groups, ga, be, eps, kind)[0] * w).sum())

    _, mean, rstd, _ = T.norm_forward(x, groups, ga, be, eps, kind)
    grads, _ = T.norm_backward(w, x, mean, rstd, groups, ga, be, kind)
    for which, (arg, grad) in enumerate(zip((x, ga, be), grads)):
        for idx in np.ndindex(arg.shape):
            up, down = ([a.copy() for a in (x, ga, be)] for _ in range(2))
            up[which][idx] += h
            down[which][idx] -= h
            assert abs((loss(*up) - loss(*down)) / (2 * h) - grad[idx]) < 1e-6


def test_adamw_is_torchs_on_kept_elements():
    rng = np.random.default_rng(2)
    w = torch.from_numpy(rng.standard_normal((4, 3, 3, 3))).requires_grad_(True)
    taps = np.array([0x0B8, 0, 0x017, 0x1FF] * 3)
    p, m, v = w.detach().numpy().reshape(-1).copy(), np.zeros(108), np.zeros(108)
    opt = torch.optim.AdamW([w], lr=0.01, betas=(0.8, 0.95), eps=1e-6, weight_decay=0.1)
    k = T.kept(taps, 108)
    for step in range(1, 6):
        g = rng.standard_normal(108)
        w.grad = torch.from_numpy(g.reshape(w.shape))
        opt.step()
        p, m, v = T.adamw(p, g, m, v, taps, 0.01, 0.8, 0.95, 1e-6, 0.1, step)
    np.testing.assert_allclose(p[k], w.detach().numpy().reshape(-1)[k], rtol=1e-12)
    assert k.sum() == 3 * (4 + 0 + 4 + 9) and not m[~k].any()


def test_eight_bit_values_are_float8_and_neighbours():
    rng = np.random.default_rng(3)
    t = rng.standard_normal(4 * T.BLOCK) * np.repeat([1e-9, 1.0, 3e4, 0.0], T.BLOCK)
    r = rng.integers(0, 65536, t.size)
    w, scale, _ = T.encode(t, r, False)
    as8 = torch.from_numpy(w).to(torch.float8_e4m3fn).double().numpy()
    np.testing.assert_array_equal(w, as8)                          # every value is one of the format's
    step = 2.0 ** (np.floor(np.log2(np.maximum(np.abs(t / scale), 2.0 ** -6))) - 3)
    assert np.all(np.abs(w - t / scale) <= step)
    assert np.all(np.abs(w) <= 448) and np.all(np.frexp(scale)[0] == 0.5)
    tops = np.abs((t / scale).reshape(-1, T.BLOCK)).max(1)[:3]
    assert np.all((tops > 224) & (tops <= 448))


def test_eight_bit_second_moments_stay_above_zero():
    t = np.full(T.BLOCK, 1e-12)
    t[0], t[1] = 1.0, 0.0
    w, _, _ = T.encode(t, np.zeros(T.BLOCK, np.int64), True)
    assert w[1] == 0 and np.all(w[2:] == 2.0 ** -9)


def test_dither_is_uniform_and_changes_with_the_step():
    """Means of n uniform values are within 4 sigma, 4 / sqrt(12 n) of the range; pairs are uncorrelated
    within 4 / sqrt(n); rounding with it has no bias."""
    n = 1 << 18
    m, v = T.dither(7, 3, 0, n)
    m2, v2 = T.dither(7, 4, 0, n)
    for a in (m, v, m2, v2):
        assert abs(a.mean() / 65535 - 0.5) < 4 / math.sqrt(12 * n)
    for a, b in ((m, v), (m, m2), (v, v2), (v[:-1], v[1:]), (v[:-8], v[8:])):
        assert abs(np.corrcoef(a, b)[0, 1]) < 4 / math.sqrt(len(a))
    np.testing.assert_array_equal(T.dither(7, 3, 256, 512)[1], v[256:768])
    t = np.full(n, 0.9)
    w, scale, _ = T.encode(t, v, True)                             # 0.9 lies at 0.6 of a step
    assert abs((w * scale).mean() - 0.9) < 4 * 0.0625 * math.sqrt(0.24 / n) + 0.0625 / 131072


# ------------------------------------------------------------------------------------ refusals

def test_group_norm_refusals(lib):
    p = ctypes.c_void_p
    size = ctypes.c_size_t()

    def fwd(x=256, px=8, sx=32, dt=0, n=1, hw=4, c=8, g=2, ga=None, be=None, eps=1e-5, act=0, y=4096, mean=None, rstd=None,
            ws=8192, wsb=1 << 20):
        return lib.pp_group_norm(p(x) if x else None, px, sx, dt, n, hw, c, g, p(ga) if ga else None, p(be) if be else None, eps,
                                 act, p(y) if y else None, p(mean) if mean else None, None, p(ws) if ws else None, wsb, None)

    assert fwd(dt=3) == DTYPE and fwd(dt=-1) == DTYPE
    for bad in (dict(n=-1), dict(hw=-1), dict(c=0), dict(g=0), dict(g=3), dict(c=1 << 21, g=1), dict(n=65535), dict(px=7),
                dict(n=2, sx=-8), dict(n=60000, hw=1 << 30, c=1 << 20)):
        assert fwd(**bad) == SHAPE, bad
    assert fwd(act=3) == ARG and fwd(eps=-1.0) == ARG and fwd(eps=float("nan")) == ARG and fwd(eps=math.inf) == ARG
    assert fwd(x=0) == NULL and fwd(y=0) == NULL and fwd(ws=0) == NULL
    assert fwd(x=257) == ALIGN and fwd(x=258) == ALIGN and fwd(y=4097) == ALIGN and fwd(ga=3) == ALIGN and fwd(ws=8200) == ALIGN
    assert fwd(mean=6) == ALIGN
    assert fwd(wsb=4) == BUFFER
    assert fwd(y=256 + 64) == BUFFER                              # y inside x
    assert fwd(y=256, px=16, sx=64) == BUFFER                     # in place needs a dense x
    assert fwd(n=0, x=0) == 0 and fwd(hw=0, y=0) == 0
    assert lib.pp_group_norm_workspace_size(0, 1, 4, 8, 2, 2, ctypes.byref(size)) == ARG
    assert lib.pp_group_norm_workspace_size(0, 1, 4, 8, 3, 0, ctypes.byref(size)) == SHAPE
    assert lib.pp_group_norm_workspace_size(0, 1, 4, 8, 2, 0, None) == NULL

    def bwd(dy=256, x=1024, mean=64, rstd=64, dx=4096, act=0, wsb=1 << 20, dtype=0, dgamma=None):
        f = lambda v: p(v) if v else None  # noqa: E731
        return lib.pp_group_norm_backward(f(dy), 8, 32, f(x), 8, 32, dtype, 1, 4, 8, 2, None, None, f(mean), f(rstd), act, f(dx),
                                          f(dgamma), None, p(8192), wsb, None)

    assert bwd(dy=0) == NULL and bwd(x=0) == NULL and bwd(mean=0) == NULL and bwd(rstd=0) == NULL and bwd(dx=0) == NULL
    assert bwd(dtype=9) == DTYPE and bwd(act=-1) == ARG and bwd(wsb=0) == BUFFER and bwd(dgamma=2) == ALIGN
    assert bwd(dx=1024) == BUFFER and bwd(dx=256 + 32) == BUFFER


def _create(lib, numel, dtypes, taps=None, params=None, copies=None, copy_dtype=1, decay=None):
    n = len(numel)
    h = ctypes.c_void_p()
    arr = lambda v: (ctypes.c_void_p * n)(*v) if v is not None else None  # noqa: E731
    st = lib.pp_tensors_create(n, (ctypes.c_int64 * n)(*numel), (ctypes.c_int * n)(*dtypes), arr(taps), arr(params), arr(copies),
                               copy_dtype, (ctypes.c_float * n)(*decay) if decay is not None else None, ctypes.byref(h))
    return st, h


def test_tensors_refusals(lib):
    assert _create(lib, [-1], [0])[0] == SHAPE and _create(lib, [8], [3])[0] == DTYPE
    assert _create(lib, [8], [0], taps=[64])[0] == SHAPE and _create(lib, [9], [0], taps=[65])[0] == ALIGN
    assert _create(lib, [8], [0], params=[None])[0] == NULL and _create(lib, [8], [0], params=[66])[0] == ALIGN
    assert _create(lib, [8], [0], copies=[64], copy_dtype=0)[0] == DTYPE and _create(lib, [8], [0], copies=[65])[0] == ALIGN
    assert _create(lib, [8], [0], decay=[math.nan])[0] == ARG
    assert lib.pp_tensors_create(1, None, None, None, None, None, 1, None, ctypes.byref(ctypes.c_void_p())) == NULL
    assert lib.pp_tensors_create(-1, None, None, None, None, None, 1, None, ctypes.byref(ctypes.c_void_p())) == SHAPE

    st, h = _create(lib, [10, 0, 513], [0, 1, 2], params=[256, None, 4096])
    assert st == 0
    v = ctypes.c_int64()
    got = []
    for key in (0, 2, 16, 17, 18):
        assert lib.pp_tensors_query(h, key, ctypes.byref(v)) == 0
        got.append(v.value)
    assert got == [3, 256 + 768, 0, 256, 256]
    assert lib.pp_tensors_query(h, 19, ctypes.byref(v)) == ARG and lib.pp_tensors_query(h, 3, ctypes.byref(v)) == ARG
    assert lib.pp_tensors_query(None, 0, ctypes.byref(v)) == NULL
    grads = (ctypes.c_void_p * 3)(256, None, 4096)
    step = lambda bits=32, lr=1e-3, b1=0.9, b2=0.999, eps=1e-8, t=1, m=256, gs=None: lib.pp_adamw_step(  # noqa: E731
        h, grads, bits, ctypes.c_void_p(m) if m else None, ctypes.c_void_p(512), None, None, lr, b1, b2, eps, t, 0,
        ctypes.c_void_p(gs) if gs else None, None)
    assert step() == NOT_BOUND and lib.pp_grad_norm(h, grads, 1.0, ctypes.c_void_p(64), None) == NOT_BOUND
    assert lib.pp_tensors_bind(h, None, 1 << 20, None) == NULL
    assert lib.pp_tensors_bind(h, ctypes.c_void_p(256), 8, None) == BUFFER
    assert lib.pp_tensors_bind(h, ctypes.c_void_p(272), 1 << 20, None) == ALIGN
    assert lib.pp_grad_norm(None, grads, 1.0, ctypes.c_void_p(64), None) == NULL
    assert lib.pp_tensors_destroy(h) == 0 and lib.pp_tensors_destroy(None) == 0


def test_bindings_refuse_what_is_not_on_the_gpu():
    x = torch.zeros(1, 8, 2, 2).contiguous(memory_format=torch.channels_last)
    with pytest.raises(ValueError, match="CUDA"):
        norm.pp_group_norm(x, 2)
    with pytest.raises(ValueError, match="CUDA"):
        norm.pp_group_norm_backward(x, x, x, x, 2)
    with pytest.raises(ValueError, match="CUDA"):
        optim.AdamW([torch.zeros(4)])
    with pytest.raises(ValueError):
        optim.AdamW([])
    with pytest.raises(ValueError):
        optim.AdamW([torch.zeros(4)], state_bits=16)
    with pytest.raises(ValueError):
        optim.GradNorm([(4,)], device="cpu")


def test_strides_of_channels_last_tensors():
    base = torch.zeros(3, 5, 7, 12)                                # [N, H, W, wide]
    x = base.permute(0, 3, 1, 2)
    assert norm._strides(x) == (12, 420)
    assert norm._strides(x[:, 2:6]) == (12, 420)                   # a range of channels
    assert norm._strides(x[::2]) == (12, 840)                      # every other sample
    assert norm._strides(x[:, :, :, 1:5]) is None                  # rows that do not join up
    assert norm._strides(torch.zeros(3, 12, 5, 7)) is None
    assert norm._strides(torch.zeros(3, 1, 5, 7)) == (1, 35)       # one channel is both orders
    assert norm._strides(torch.zeros(3, 12, 1, 1)) == (12, 12)
    assert norm._strides(torch.zeros(1, 4, 1, 1).expand(5, 4, 1, 1)) == (4, 0)


def test_taps_of_a_pruned_weight():
    w = torch.zeros(2, 2, 3, 3)
    w[0, 1, 0, 0] = 1.0
    w[1, 0].view(-1)[[3, 4, 5, 7]] = -2.0
    assert optim.taps_of(w).tolist() == [0, 1, 0x0B8, 0] and optim.taps_of(w).dtype == torch.int16
    with pytest.raises(ValueError):
        optim.taps_of(torch.zeros(2, 2, 5, 5))


@pytest.mark.parametrize("masked", [False, True])
def test_a_handle_for_the_norm_alone_has_no_table_of_steps(lib, masked):
    """32 bytes for every 16384 elements and the partial sums of a launch; with parameters 64 for every 2048 too."""
    numel, v = [512 * 512 * 9] * 24 + [10, 0], ctypes.c_int64()
    taps = [1 << 20] * 24 + [None, None] if masked else None
    sums = 512 + 152 * 5 * 8
    got = []
    for params in (None, [(i + 1) << 30 for i in range(26)]):
        st, h = _create(lib, numel, [0] * 26, taps=taps, params=params)
        assert st == 0 and lib.pp_tensors_query(h, 1, ctypes.byref(v)) == 0
        got.append(v.value)
        assert lib.pp_tensors_query(h, 2, ctypes.byref(v)) == 0 and v.value == 24 * 512 * 512 * 9 + 256
        lib.pp_tensors_destroy(h)
    spans, chunks = 24 * 144 + 1, 24 * 1152 + 1
    assert got[0] <= 32 * spans + 256 + sums and got[1] >= 64 * chunks + 32 * spans + sums


def test_parameters_and_copies_that_share_memory_are_refused(lib):
    """A step would write them in no order."""
    both = [0, 0]
    for kw in (dict(params=[4096, 4096]), dict(params=[4096, 4096 + 36]), dict(params=[4096 + 36, 4096]),
               dict(params=[4096, 8192], copies=[1024, 1024 + 18]), dict(params=[4096, 8192], copies=[None, 4096 + 32]),
               dict(params=[4096, 8192], copies=[8192, None])):
        assert _create(lib, [10, 10], both, **kw)[0] == BUFFER, kw
    for kw in (dict(params=[4096, 4096 + 40]), dict(params=[4096, 8192], copies=[4096 + 40, 4096 - 20])):
        st, h = _create(lib, [10, 10], both, **kw)
        assert st == 0 and lib.pp_tensors_destroy(h) == 0
    st, h = _create(lib, [10, 0], both, params=[4096, 4096])      # of no elements
    assert st == 0 and lib.pp_tensors_destroy(h) == 0

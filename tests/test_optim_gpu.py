"""The gradients' norm and AdamW steps on the GPU against the float64 oracle."""
import math

import numpy as np
import pytest
import torch

from oracle import train as T
from paper_2003_06513_gb300 import optim
from paper_2003_06513_gb300._lib import PatconvError

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
E = 2.0 ** -24
HYPER = dict(lr=1e-2, b1=0.9, b2=0.99, eps=1e-6)

# element counts around a lane's eight, a block's 256 and a chunk's 2048, and 3x3 weights
SIZES = [(1,), (7,), (8,), (9,), (255,), (256,), (257,), (2047,), (2048,), (2049,), (0,), (5000,), (1, 1, 3, 3), (3, 5, 3, 3),
         (64, 32, 3, 3), (113, 1, 3, 3), (31, 33, 3, 3)]


def _taps(rng, shape):
    """Random 4-tap masks, a third of the kernels pruned away; the first and last kernels pruned."""
    if len(shape) != 4:
        return None
    t = np.array([0x0B8, 0x0B2, 0x09A, 0x03A, 0x017, 0x059, 0x134, 0x1D0, 0, 0, 0, 0x1FF], np.int16)[rng.integers(0, 12, shape[0] * shape[1])]
    if t.size > 4:
        t[0] = t[-1] = 0
    return t


def _problem(seed, masked, grad):
    rng = np.random.default_rng(seed)
    taps = [_taps(rng, s) if masked else None for s in SIZES]
    p = [(rng.standard_normal(s) * 0.1).astype(np.float32) for s in SIZES]
    for a, t in zip(p, taps):
        if t is not None:
            a.reshape(-1)[~T.kept(t, a.size)] = 0
    g = [torch.from_numpy(rng.standard_normal(s) * 10.0 ** rng.integers(-4, 2)).to(DT[grad]) for s in SIZES]
    return rng, p, g, taps


def _gpu_taps(taps):
    return [torch.from_numpy(t).cuda() if t is not None else None for t in taps]


def _close32(got, want, scale, what):
    """Within 16 fp32 roundings of the terms' sizes."""
    bad = np.abs(got - want) > 16 * E * scale + 1e-37
    assert not bad.any(), f"{what}: {bad.sum()} of {bad.size}"


@pytest.mark.parametrize("masked", [False, True])
@pytest.mark.parametrize("grad", ["f32", "f16", "bf16"])
def test_steps_with_fp32_states(grad, masked):
    rng, p, g, taps = _problem(1, masked, grad)
    decay = [0.1 if len(s) == 4 else 0.0 for s in SIZES]
    params = [torch.from_numpy(a).cuda() for a in p]
    opt = optim.AdamW(params, HYPER["lr"], (HYPER["b1"], HYPER["b2"]), HYPER["eps"], decay, taps=_gpu_taps(taps), grad_dtypes=DT[grad])
    scale = torch.tensor([0.75], device="cuda")
    for step in (1, 2, 3):
        before = [a.double().cpu().numpy().reshape(-1) for a in params]
        states = [[a.double().cpu().numpy() for a in opt.state_of(i)] for i in range(len(SIZES))]
        opt.step([a.cuda() for a in g], grad_scale=scale)
        for i, t in enumerate(taps):
            gi = g[i].double().numpy().reshape(-1) * 0.75
            m, v = states[i]
            want_p, want_m, want_v = T.adamw(before[i], gi, m, v, t, step=step, decay=decay[i], **HYPER)
            got_m, got_v = (a.double().cpu().numpy() for a in opt.state_of(i))
            _close32(got_m, want_m, np.abs(m) + np.abs(gi), "m")
            _close32(got_v, want_v, v + gi * gi, "v")
            # the quotient is off by its terms' roundings, relative to |m| + |g| over the root
            den = np.sqrt(want_v / (1 - HYPER["b2"] ** step)) + HYPER["eps"]
            u = HYPER["lr"] * (np.abs(m) + np.abs(gi)) / (1 - HYPER["b1"] ** step) / den
            _close32(params[i].double().cpu().numpy().reshape(-1), want_p, np.abs(before[i]) + u, "p")
        g = [torch.from_numpy(rng.standard_normal(s)).to(DT[grad]) for s in SIZES]


@pytest.mark.parametrize("masked", [False, True])
@pytest.mark.parametrize("grad", ["f32", "bf16"])
def test_steps_with_8_bit_states(grad, masked):
    """Values over their scales equal the oracle's, but where rounding turns within the reach of fp32
    errors (margin): there they may be its neighbour."""
    rng, p, g, taps = _problem(2, masked, grad)
    params = [torch.from_numpy(a).cuda() for a in p]
    opt = optim.AdamW(params, HYPER["lr"], (HYPER["b1"], HYPER["b2"]), HYPER["eps"], 0.1, state_bits=8, taps=_gpu_taps(taps),
                      grad_dtypes=DT[grad], seed=77)
    at = np.cumsum([0] + [-(-math.prod(s) // 256) * 256 for s in SIZES])
    for step in (1, 2, 3):
        before = [a.double().cpu().numpy().reshape(-1) for a in params]
        states = [[a.double().cpu().numpy() for a in opt.state_of(i)] for i in range(len(SIZES))]
        opt.step([a.cuda() for a in g])
        rm, rv = T.dither(77, step, 0, int(at[-1]))
        for i, t in enumerate(taps):
            gi = g[i].double().numpy().reshape(-1)
            m, v = states[i]
            want_p, want_m, want_v = T.adamw(before[i], gi, m, v, t, step=step, decay=0.1, **HYPER)
            den = np.sqrt(want_v / (1 - HYPER["b2"] ** step)) + HYPER["eps"]
            u = HYPER["lr"] * (np.abs(m) + np.abs(gi)) / (1 - HYPER["b1"] ** step) / den
            _close32(params[i].double().cpu().numpy().reshape(-1), want_p, np.abs(before[i]) + u, "p")
            sl, blocks = slice(at[i], at[i + 1]), slice(at[i] // 256, at[i + 1] // 256)
            for name, want, r, positive in (("m", want_m, rm, False), ("v", want_v, rv, True)):
                full = np.zeros(at[i + 1] - at[i])
                full[:want.size] = want
                w, scale, margin = T.encode(full, r[sl], positive)
                code = getattr(opt, name)[sl].double().cpu().numpy()
                got_scale = getattr(opt, name + "_scale")[blocks].double().cpu().numpy()
                if full.size:
                    np.testing.assert_array_equal(got_scale, scale[::256])
                # fp32's error of the sum, in steps of the code: relative to the terms, not to the sum
                terms = np.zeros_like(full)
                terms[:want.size] = (np.abs(m) + np.abs(gi)) if name == "m" else v + gi * gi
                step_size = 2.0 ** (np.floor(np.log2(np.maximum(np.abs(full) / scale, 2.0 ** -6))) - 3)
                reach = 16 * E * terms / scale / step_size + 1e-6
                wrong = (code != w) & ~((margin <= reach) & (np.abs(code - w) <= 2 * step_size))
                assert not wrong.any(), (name, i, wrong.sum())
        g = [torch.from_numpy(rng.standard_normal(s) * 10.0 ** rng.integers(-4, 2)).to(DT[grad]) for s in SIZES]


def test_unaligned_tensors():
    """Parameters, gradients and copies at odd addresses give what aligned ones give."""
    shape, n = (16, 16, 3, 3), 2304
    taps = optim.taps_of((torch.rand(shape) > 0.5).float().cuda())
    for bits in (32, 8):
        for dtype in (torch.float32, torch.bfloat16):
            torch.manual_seed(3)
            start, grad = torch.randn(n, device="cuda"), torch.randn(n, device="cuda").to(dtype)
            got = []
            for shift in (0, 1, 3):
                p = torch.empty(n + 8, device="cuda")[shift:shift + n].copy_(start).view(shape)
                c = torch.empty(n + 8, device="cuda", dtype=torch.float16)[shift:shift + n].copy_(start).view(shape)
                g = torch.empty(n + 8, device="cuda", dtype=dtype)[shift:shift + n].copy_(grad).view(shape)
                opt = optim.AdamW([p], state_bits=bits, taps=[taps], grad_dtypes=dtype, copies=[c])
                norm, _ = opt.grad_norm([g], 1.0)
                opt.step([g])
                opt.step([g])
                got.append((p.clone(), c.clone(), opt.m.view(torch.uint8), opt.v.view(torch.uint8), norm))
            for other in got[1:]:
                assert all(torch.equal(a, b) for a, b in zip(got[0], other))
            assert torch.equal(got[0][1], got[0][0].half())


@pytest.mark.parametrize("bits", [32, 8])
def test_masked_places_are_left_alone_whatever_their_gradient(bits):
    torch.manual_seed(4)
    w = torch.randn(40, 24, 3, 3, device="cuda")
    w *= (torch.rand_like(w) > 0.6) & (torch.rand(40, 24, 1, 1, device="cuda") > 0.5)
    pruned = w == 0
    good = torch.randn_like(w)
    bad = torch.where(pruned, torch.tensor([float("nan"), float("inf"), -3e38], device="cuda")[torch.randint(0, 3, w.shape, device="cuda")], good)
    results = []
    for g in (good, bad):
        p = w.clone()
        opt = optim.AdamW([p], taps=[optim.taps_of(w)], state_bits=bits, weight_decay=0.1)
        norm, scale = opt.grad_norm([g], 0.5)
        for _ in range(3):
            opt.step([g], grad_scale=scale)
        assert not p[pruned].any() and (p != w)[~pruned].all()
        assert not opt.state_of(0)[0].view(w.shape)[pruned].any()
        results.append((p, norm, opt.m.view(torch.uint8), opt.v.view(torch.uint8)))
    assert all(torch.equal(a, b) for a, b in zip(*results))


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_what_is_not_finite_stays_at_its_place(bits, bad):
    torch.manual_seed(5)
    g = torch.randn(1000, device="cuda")
    runs = []
    for spoil in (False, True):
        p, gi = torch.ones(1000, device="cuda"), g.clone()
        if spoil:
            gi[300] = bad
        opt = optim.AdamW([p], state_bits=bits)
        opt.step([gi])
        opt.step([g])
        runs.append((p, *opt.state_of(0)))
    keep = torch.arange(1000, device="cuda") != 300
    for clean, spoilt in zip(*runs):
        assert torch.equal(clean[keep], spoilt[keep])
    assert torch.isnan(runs[1][0][300]) and not torch.isfinite(runs[1][1][300])


def test_tensors_without_a_gradient_and_many_tensors():
    """More tensors than a launch takes; every third has no gradient and stays."""
    torch.manual_seed(6)
    for count in (3, 64, 65, 448, 449, 1000):
        start = [torch.randn(1 + i % 50, device="cuda") for i in range(count)]
        grads = [None if i % 3 == 0 else torch.randn_like(a) for i, a in enumerate(start)]
        params = [a.clone() for a in start]
        opt = optim.AdamW(params, lr=0.1, weight_decay=0.0)
        norm, scale = opt.grad_norm(grads, 1.0)
        opt.step(grads)
        flat = torch.cat([g for g in grads if g is not None]).double()
        assert float(norm) == pytest.approx(float(flat.norm()), rel=1e-6)
        assert float(scale) == pytest.approx(min(1.0, 1 / float(flat.norm())), rel=1e-6)
        for a, b, g in zip(start, params, grads):
            if g is None:
                assert torch.equal(a, b)
            else:       # the first step is lr times the gradient's sign, but for eps
                assert torch.allclose(b, a - 0.1 * g / (g.abs() + 1e-8), rtol=1e-5, atol=1e-6)


def test_eight_bit_moments_follow_a_steady_gradient():
    """With a constant gradient m tends to g and v to g^2 and their averages stay there: rounding has no
    bias.  A v's own noise is about 0.1 sqrt(step (1 - b2) / (2 (1 - b2))) of it, 22 %; the mean of 2^16
    is then known to 0.1 %, m's to less."""
    g = torch.full((1 << 16,), 3e-3, device="cuda") * torch.linspace(0.5, 1.0, 1 << 16, device="cuda")
    p = torch.zeros_like(g)
    opt = optim.AdamW([p], state_bits=8, betas=(0.9, 0.99))
    for _ in range(1500):
        opt.step([g])
    m, v = opt.state_of(0)
    assert abs(float((m / g).mean()) - 1) < 0.005
    assert abs(float((v / (g * g)).mean()) - 1) < 0.01
    for _ in range(1500):                                # and they decay when it stops
        opt.step([torch.zeros_like(g)])
    assert float(opt.state_of(0)[1].mean()) < 1e-3 * float((g * g).mean())


@pytest.mark.parametrize("bits", [32, 8])
def test_state_dict_resumes_with_the_same_bits(bits):
    torch.manual_seed(7)
    grads = [[torch.randn(700, device="cuda"), torch.randn(9, 4, 3, 3, device="cuda")] for _ in range(4)]
    p = [torch.zeros(700, device="cuda"), torch.zeros(9, 4, 3, 3, device="cuda")]
    opt = optim.AdamW(p, state_bits=bits, seed=5)
    for g in grads[:2]:
        opt.step(g)
    q = [a.clone() for a in p]
    saved = {k: a.clone() if torch.is_tensor(a) else a for k, a in opt.state_dict().items()}
    resumed = optim.AdamW(q, state_bits=bits, seed=5, state=saved)
    for g in grads[2:]:
        opt.step(g)
        resumed.step(g)
    assert all(torch.equal(a, b) for a, b in zip(p, q)) and opt.steps == resumed.steps == 4
    assert torch.equal(opt.m.view(torch.uint8), resumed.m.view(torch.uint8))


def test_grads_of_parameters_other_orders_streams_and_graphs():
    torch.manual_seed(8)
    w = torch.randn(8, 4, 5, 5, device="cuda").contiguous(memory_format=torch.channels_last).requires_grad_(True)
    b = torch.randn(8, device="cuda", requires_grad=True)
    x = torch.randn(2, 4, 9, 9, device="cuda").contiguous(memory_format=torch.channels_last)
    ref = [a.detach().clone().requires_grad_(True) for a in (w, b)]
    opt, want = optim.AdamW([w, b], lr=0.01, weight_decay=0.1), torch.optim.AdamW(ref, lr=0.01, weight_decay=0.1)
    for _ in range(3):
        for ps, o in (((w, b), opt), (ref, want)):
            for a in ps:
                a.grad = None
            torch.nn.functional.conv2d(x, *ps).square().mean().backward()
        for a, c in zip((w, b), ref):
            c.grad.copy_(a.grad)
        version = w._version
        opt.step()
        want.step()
        assert w._version > version
    assert all(torch.allclose(a, c, rtol=1e-6, atol=1e-7) for a, c in zip((w, b), ref))

    p, g = torch.zeros(5000, device="cuda"), torch.randn(5000, device="cuda")
    s = torch.cuda.Stream()
    opt = optim.AdamW([p], state_bits=8, stream=s)
    s.wait_stream(torch.cuda.current_stream())
    norm, scale = opt.grad_norm([g], 1.0, stream=s)
    opt.step([g], grad_scale=scale, stream=s)
    s.synchronize()
    q = torch.zeros_like(p)
    other = optim.AdamW([q], state_bits=8)
    out = torch.empty(2, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        norm2, scale2 = other.grad_norm([g], 1.0, out=out)
        other.step([g], grad_scale=scale2)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(p, q) and torch.equal(norm, norm2) and torch.equal(opt.m.view(torch.uint8), other.m.view(torch.uint8))


@pytest.mark.parametrize("grad", ["f32", "f16", "bf16"])
def test_grad_norm(grad):
    """Sums of squares are fp32 over at most a few hundred terms: within 2^-19 of the oracle's."""
    _, _, g, taps = _problem(9, True, grad)
    n = optim.GradNorm(SIZES, DT[grad], _gpu_taps(taps))
    dev = [a.cuda() for a in g]
    for max_norm in (1e-3, 1.0, 1e9, math.inf):
        norm, scale = n(dev, max_norm)
        want, want_scale = T.grad_norm([a.double().numpy() for a in g], taps, max_norm)
        assert float(norm) == pytest.approx(want, rel=2.0 ** -19) and float(scale) == pytest.approx(want_scale, rel=2.0 ** -18)
    assert all(torch.equal(a, b) for a, b in zip(n(dev, 1.0), n(dev, 1.0)))


@pytest.mark.parametrize("size", [1e-30, 1e-42, 1e-20, 1e19, 1e30, 3e37])
def test_grad_norm_over_the_whole_range(size):
    """Squares that fp32 does not hold."""
    torch.manual_seed(10)
    g = (torch.randn(30000, dtype=torch.float64) * size).clamp(-3.4e38, 3.4e38).float()
    want = float(g.double().norm())
    norm, scale = optim.GradNorm([(30000,)])([g.cuda()], 1.0)
    if want < 3.4e38:
        assert float(norm) == pytest.approx(want, rel=1e-5)
        assert float(scale) == pytest.approx(min(1.0, 1 / (want + 1e-6)), rel=1e-5, abs=1e-44)
    else:
        assert math.isinf(float(norm)) and float(scale) == 0


def test_grad_norm_of_nothing_zeros_and_nan():
    n = optim.GradNorm([(10,), (300, 7)])
    assert [float(a) for a in n([None, None], 1.0)] == [0.0, 1.0]
    zeros = [torch.zeros(10, device="cuda"), torch.zeros(300, 7, device="cuda")]
    assert [float(a) for a in n(zeros, 1.0)] == [0.0, 1.0]
    zeros[1][200, 3] = float("nan")
    assert all(math.isnan(float(a)) for a in n(zeros, 1.0))
    zeros[1][200, 3] = -float("inf")
    assert [float(a) for a in n(zeros, 1.0)] == [math.inf, 0.0]
    assert [float(a) for a in optim.GradNorm([])([], 1.0)] == [0.0, 1.0]


def test_refusals():
    p = torch.zeros(4, 2, 3, 3, device="cuda")
    taps = optim.taps_of(p)
    for kw in (dict(params=[p.half()]), dict(params=[p[:, :1]]), dict(params=[p, p.cpu()]), dict(taps=[taps[:4]]), dict(taps=[taps.int()]),
               dict(taps=[taps.cpu()]), dict(params=[p.contiguous(memory_format=torch.channels_last)], taps=[taps]),
               dict(params=[torch.zeros(72, device="cuda")], taps=[taps]), dict(copies=[p.double()]), dict(copies=[p.half()[:2]]),
               dict(grad_dtypes=torch.float64), dict(grad_dtypes=[torch.float32] * 2), dict(weight_decay=[0.1, 0.1])):
        with pytest.raises(ValueError):
            optim.AdamW(**(dict(params=[p]) | kw))
    opt = optim.AdamW([p], taps=[taps])
    g = torch.zeros_like(p)
    for grads in ([], [g, g], [g.half()], [g.cpu()], [g[:2]], [g.view(-1)], [torch.zeros(2, 4, 3, 3, device="cuda").transpose(0, 1)]):
        with pytest.raises(ValueError):
            opt.step(grads)
        with pytest.raises(ValueError):
            opt.grad_norm(grads, 1.0)
    for scale in (torch.ones(2, device="cuda"), torch.ones(1), torch.ones(1, device="cuda").double()):
        with pytest.raises(ValueError):
            opt.step([g], grad_scale=scale)
    for bad in (0.0, -1.0, math.nan):
        with pytest.raises(PatconvError):
            opt.grad_norm([g], bad)
    with pytest.raises(PatconvError):
        opt.step([g], lr=math.nan)
    with pytest.raises(PatconvError):
        optim.AdamW([p], betas=(1.0, 0.9)).step([g])
    assert opt.steps == 0
    with pytest.raises(ValueError):
        optim.AdamW([p], state={"m": opt.m, "v": opt.v[:8], "step": 0})
    with pytest.raises(ValueError):
        optim.AdamW([p], state_bits=8, state=opt.state_dict() | {"m_scale": None, "v_scale": None})


def test_offsets_beyond_32_bits():
    """2^31 + 300 elements in one tensor, 8-bit states: the last elements step as the first ones do."""
    if torch.cuda.mem_get_info()[0] < 40 << 30:
        pytest.skip("needs 40 GB of device memory")
    n = (1 << 31) + 300
    p, g = torch.zeros(n, device="cuda"), torch.zeros(n, dtype=torch.bfloat16, device="cuda")
    opt = optim.AdamW([p], lr=0.5, state_bits=8, grad_dtypes=torch.bfloat16, weight_decay=0.0)
    g[:300] = torch.arange(1, 301, device="cuda")
    g[-300:] = g[:300]
    norm, _ = opt.grad_norm([g], 1.0)
    opt.step([g])
    assert torch.equal(p[:300], p[-300:]) and torch.allclose(p[:300], torch.full((300,), -0.5, device="cuda"), rtol=1e-5)
    assert not p[300:-300].any()
    assert float(norm) == pytest.approx(math.sqrt(2 * sum(i * i for i in g[:300].double().tolist())), rel=1e-6)
    m, _ = opt.state_of(0)
    # the ends lie differently in their blocks: each value within an eighth of 0.1 g, a scale's grid beyond
    assert torch.allclose(m[-300:], 0.1 * g[-300:].float(), rtol=0.126, atol=0.2)


def _paths(n, rng):
    """(name, parameter of n elements, masks) that the step's kernels take by different code: whole blocks, single
    elements, masks that keep nearly all of a block and masks that keep few."""
    full = torch.full((n // 9,), 0x1FF, dtype=torch.int16, device="cuda")
    few = torch.from_numpy(rng.choice(np.array([0, 0, 0x0B8, 0x017], np.int16), n // 9)).cuda()
    for name, shift, taps in (("aligned", 0, None), ("unaligned", 1, None), ("all kept", 0, full), ("few kept", 0, few)):
        yield name, torch.zeros(n + 8, device="cuda")[shift:shift + n].view(n // 9, 1, 3, 3), taps


@pytest.mark.parametrize("grad", ["f32", "f16", "bf16"])
def test_moments_round_every_product_and_sum_in_every_path(grad):
    """fp32 moments have the bits of fp32 arithmetic with each product and sum rounded by itself."""
    rng = np.random.default_rng(12)
    n, b1, b2, f = 9 * 555, HYPER["b1"], HYPER["b2"], np.float32
    for name, p, taps in _paths(n, rng):
        opt = optim.AdamW([p], HYPER["lr"], (b1, b2), HYPER["eps"], 0.1, taps=[taps], grad_dtypes=DT[grad])
        keep = T.kept(None if taps is None else taps.cpu().numpy(), n)
        scale = torch.tensor([0.7], device="cuda")
        for step in range(5):
            g = torch.from_numpy(rng.standard_normal(n) * 10.0 ** rng.integers(-4, 2, n)).to(DT[grad])
            m, v = (a.cpu().numpy() for a in opt.state_of(0))
            opt.step([g.cuda().view(p.shape)], grad_scale=scale)
            gs = g.float().numpy() * f(scale.item())
            for got, want in zip(opt.state_of(0), (m * f(b1) + gs * f(1 - b1), v * f(b2) + (gs * gs) * f(1 - b2))):
                np.testing.assert_array_equal(got.cpu().numpy(), np.where(keep, want, 0), err_msg=f"{name}, step {step}")


@pytest.mark.parametrize("bits", [8, 32])
def test_a_step_has_the_same_bits_at_any_alignment_without_a_mask(bits):
    """Eight million elements: of 8-bit codes one in a million turns where a moment's last bit does."""
    n, got = 1 << 23, []
    for shift in (0, 1):
        gen = torch.Generator(device="cuda").manual_seed(3)
        p = torch.zeros(n + 8, device="cuda")[shift:shift + n]
        opt = optim.AdamW([p], state_bits=bits)
        for _ in range(3):
            opt.step([torch.randn(n, generator=gen, device="cuda")])
        got.append((p, opt.m.view(torch.uint8), opt.v.view(torch.uint8)))
    assert all(torch.equal(a, b) for a, b in zip(*got))


def test_grad_norm_after_a_call_that_ended_between_its_launches():
    """Such a call leaves its CTAs counted (a list of a thousand is three launches): the next one's norm is right."""
    n = optim.GradNorm([(5,)] * 1000)
    table = n._t._table
    counters = table[table.numel() - 512 - 3 * 152 * 5 * 8:][:4 * 65].view(torch.int32)
    for value in (0.5, 1.5):
        assert not counters.any()
        counters.fill_(3)
        out = torch.zeros(2, device="cuda")
        n([torch.full((5,), value, device="cuda") for _ in range(1000)], 1.0, out=out)
        assert float(out[0]) == pytest.approx(value * math.sqrt(5000), rel=1e-6)


@pytest.mark.parametrize("values", [[1.0, math.inf, 2.0, 0.0], [3e38] * 4, [1.0, -math.inf, math.inf, 3e38]], ids=str)
def test_an_infinite_norm_is_not_clipped_by_an_infinite_bound(values):
    """The default bound: the factor must not make NaN of the other gradients."""
    n, g = optim.GradNorm([(4,)]), [torch.tensor(values, device="cuda")]
    assert [float(a) for a in n(g)] == [math.inf, 1.0]
    assert [float(a) for a in n(g, 1e30)] == [math.inf, 0.0]
    p = torch.ones(4, device="cuda")
    opt = optim.AdamW([p])
    opt.step(g, grad_scale=opt.grad_norm(g)[1])
    assert torch.isfinite(p[g[0].abs() < 1e30]).all()
    g[0][0] = math.nan
    assert all(math.isnan(float(a)) for a in n(g))


def test_bias_corrections_go_by_a_tensors_own_steps():
    """Tensors whose gradients come late, or now and then, against torch.optim.AdamW: fp32 steps of 0.01, each right to
    some roundings of a parameter near 1."""
    torch.manual_seed(9)
    start = [torch.randn(300, device="cuda") for _ in range(4)]
    p, q = [a.clone() for a in start], [a.clone().requires_grad_(True) for a in start]
    opt, ref = optim.AdamW(p, lr=0.01, weight_decay=0.1), torch.optim.AdamW(q, lr=0.01, weight_decay=0.1)
    for step in range(24):
        if step == 15:
            opt = optim.AdamW(p, lr=0.01, weight_decay=0.1, state=opt.state_dict())
        g = [torch.randn(300, device="cuda") if on else None for on in (True, step >= 12, step % 2, step == 20)]
        for a, b in zip(q, g):
            a.grad = b
        opt.step(g)
        ref.step()
    assert opt.steps == 24 and opt.state_dict()["missed"] == [0, 12, 12, 23]
    assert all(torch.allclose(a, b, rtol=1e-5, atol=1e-6) for a, b in zip(p, q))
    for bad in ([0, 0], [0, 0, 0, -1]):
        with pytest.raises(ValueError, match="missed"):
            optim.AdamW(p, state=opt.state_dict() | {"missed": bad})
    with pytest.raises(ValueError, match="missed"):
        optim.AdamW(p, state=opt.state_dict() | {"missed": [0, 0, 0, 25]}).step(g[:3] + [torch.zeros(300, device="cuda")])


@pytest.mark.parametrize("bits", [8, 32])
def test_a_tensor_that_comes_late_steps_as_it_would_alone(bits):
    torch.manual_seed(10)
    start = torch.randn(3000, device="cuda")
    x, y, alone = start.clone(), torch.zeros(50, device="cuda"), start.clone()
    both, one = optim.AdamW([x, y], state_bits=bits, seed=3), optim.AdamW([alone], state_bits=bits, seed=3)
    for step in range(9):
        g = torch.randn(3000, device="cuda") if step > 4 else None
        both.step([g, torch.randn(50, device="cuda") if step != 7 else None])
        if g is not None:
            one.step([g])
    assert torch.equal(x, alone) and all(torch.equal(a, b) for a, b in zip(both.state_of(0), one.state_of(0)))

"""What is measured: the operators of masked retraining of a pattern-pruned network.

Between the pruned 3x3 convolutions a network being retrained runs group norm with its activation
(channels last, forward and backward); after the backward pass the optimiser takes the norm of all
gradients (clipping) and an AdamW step over all tensors, in which the pruned taps stay as they are.

* ``group_norm``: y = act(gamma_c (x - mean) rstd + beta_c), mean and rstd over a group's channels
  and all pixels of a sample; act is the identity, ReLU or SiLU.  A training program keeps mean and
  rstd for the backward pass, which returns dx, dgamma and dbeta.
* ``adamw``: m = b1 m + (1 - b1) g, v = b2 v + (1 - b2) g^2, p = p (1 - lr wd) - lr (m / (1 - b1^t))
  / (sqrt(v / (1 - b2^t)) + eps), g being the gradient times a factor that the device holds.  The
  states are fp32, or 8-bit floats (e4m3) times a power of two for every 256 elements, rounded with
  a dither that is a function of the step's key and the element's position.
* ``grad_norm``: the root of the sum of squares over all kept gradients, and the clip factor.

Sizes are those of this repository's networks (VGG-16, ResNet-50's 3x3 convolutions, MobileNet-V2's
depthwise layers), odd sizes between them, and generic wide layers.
"""
from __future__ import annotations

import math

import torch

own = False

DT = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
SIZE = {"f32": 4, "f16": 2, "bf16": 2}
EPS = 1e-5
B1, B2, ADAM_EPS, LR, DECAY = 0.9, 0.999, 1e-8, 1e-3, 0.05
BLOCK = 256                 # elements that share a scale; a tensor's states start at a multiple of it
LARGEST_BYTES = 2 ** 30     # of a drawn case


# --------------------------------------------------------------------------------------- cases

def _norm(name, kind, n, c, g, h, w, act, dtype):
    return {"name": name, "kind": kind, "n": n, "c": c, "g": g, "h": h, "w": w, "act": act, "dtype": dtype}


def _many(name, kind, net, keep, grad, bits=32):
    return {"name": name, "kind": kind, "net": net, "keep": keep, "grad": grad, "bits": bits}


def listed():
    return [
        # one small sample, the framework's single layer: launch and latency
        _norm("norm_32_n1", "forward", 1, 64, 8, 32, 32, "relu", "f32"),
        # the middle of a network in half precision, ordinary batch
        _norm("norm_56_n32_f16", "forward", 32, 256, 32, 56, 56, "silu", "f16"),
        # the first block: the largest maps, two channels a group
        _norm("norm_224_n32", "forward", 32, 64, 32, 224, 224, "relu", "f32"),
        # ragged: odd channels a group, an odd map, rows that are no multiple of 16 bytes
        _norm("norm_back_ragged", "backward", 5, 150, 10, 45, 61, "silu", "bf16"),
        # late layers: small maps, many channels
        _norm("norm_back_14_n32", "backward", 32, 512, 32, 14, 14, "relu", "f32"),
        # the second block's gradient in half precision
        _norm("norm_back_112_n32_f16", "backward", 32, 128, 32, 112, 112, "silu", "f16"),
        # many small tensors, nothing pruned away but the taps: launch and latency
        _many("adamw_mobilenet", "adamw", "mobilenet", 1.0, "f32"),
        # the pruned VGG-16 stack with its norms' parameters
        _many("adamw_vgg16", "adamw", "vgg16", 0.3, "f32"),
        # ResNet-50's 3x3 layers, 8-bit states, half-precision gradients
        _many("adamw8_resnet50_bf16", "adamw", "resnet50", 0.4, "bf16", 8),
        # wide layers before anything is pruned: the largest step
        _many("adamw8_wide", "adamw", "wide24", 0.0, "f32", 8),
        # clipping: the pruned ResNet-50 layers' gradients, and the wide layers' in half precision
        _many("grad_norm_resnet50", "grad_norm", "resnet50", 0.4, "f32"),
        _many("grad_norm_wide_bf16", "grad_norm", "wide24", 0.0, "bf16"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    while True:
        if rng.random() < 0.55:
            g = rng.choice([1, 2, 4, 8, 10, 16, 32, 32, 32, 64])
            c = g * _log(rng, 1, 64)
            h = _log(rng, 7, 224)
            w = h if rng.random() < 0.5 else max(7, min(224, int(h * rng.uniform(0.6, 1.6))))
            case = _norm("", rng.choice(["forward", "backward"]), _log(rng, 1, 64), c, g, h, w,
                         rng.choice(["none", "relu", "silu"]), rng.choice(["f32", "f16", "bf16"]))
            fits = 2 <= c <= 1024
        else:
            net = rng.choice(["mobilenet", "resnet50", "vgg16", "wide", "odd", "odd"])
            net = f"wide{rng.randint(1, 20)}" if net == "wide" else f"odd{rng.randint(1, 9999)}" if net == "odd" else net
            keep = rng.choice([0.0, 0.25, 0.3, 0.4, 0.5, 1.0])   # 0: nothing is masked
            kind = "adamw" if rng.random() < 0.7 else "grad_norm"
            case = _many("", kind, net, keep, rng.choice(["f32", "f16", "bf16"]),
                         rng.choice([32, 8]) if kind == "adamw" else 32)
            fits = True
        del case["name"]
        if fits and work(case)["bytes"] <= LARGEST_BYTES:
            return case


# ------------------------------------------------------------------------------------ the inputs

VGG16 = [(3, 64), (64, 64), (64, 128), (128, 128), (128, 256), (256, 256), (256, 256), (256, 512),
         (512, 512), (512, 512), (512, 512), (512, 512), (512, 512)]
RESNET50 = [64] * 3 + [128] * 4 + [256] * 6 + [512] * 3
MOBILENET = [32, 96, 144, 144, 192, 192, 192, 384, 384, 384, 384, 576, 576, 576, 960, 960, 960]
# the default library: centre + 3 of the 4 edge neighbours, centre + an edge and its two corners
PATTERNS = [0x0B8, 0x0B2, 0x09A, 0x03A, 0x017, 0x059, 0x134, 0x1D0]


def _shapes(net):
    """Shapes of a network's tensors: per layer the 3x3 weights and its norm's gamma and beta."""
    if net == "vgg16":
        convs = [(co, ci) for ci, co in VGG16]
    elif net == "resnet50":
        convs = [(c, c) for c in RESNET50]
    elif net == "mobilenet":
        convs = [(c, 1) for c in MOBILENET]
    elif net.startswith("wide"):
        convs = [(512, 512)] * int(net[4:])
    else:                                      # odd sizes, from one to ten layers
        k = int(net[3:])
        convs = [(1 + (k * (17 + 6 * i)) % 211, 1 + (k * (29 + 10 * i)) % 173) for i in range(1 + k % 10)]
    shapes = []
    for co, ci in convs:
        shapes += [(co, ci, 3, 3)] + ([(co,), (co,)] if len(convs) <= 20 else [])
    return shapes


def _masked(shape, case):
    return case["keep"] > 0 and len(shape) == 4


def _kernels_kept(shape, keep):
    return max(1, min(shape[0] * shape[1], math.floor(keep * shape[0] * shape[1] + 0.5)))


def prepare(case, seed):
    return _prepare_norm(case, seed) if "act" in case else _prepare_many(case, seed)


def _prepare_norm(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    n, c, g, h, w, dt = case["n"], case["c"], case["g"], case["h"], case["w"], DT[case["dtype"]]

    def normal(*shape, dtype=torch.float32):
        return torch.randn(*shape, generator=gen, device="cuda", dtype=dtype)

    # a convolution's outputs: every channel with its own mean and spread
    x = normal(n, h, w, c, dtype=dt).mul_((0.5 + normal(c).abs()).to(dt)).add_((0.3 * normal(c)).to(dt))
    state = {"case": case, "x": x.permute(0, 3, 1, 2), "gamma": 1 + 0.1 * normal(c), "beta": 0.1 * normal(c)}
    if case["kind"] == "backward":
        state["dy"] = (normal(n, h, w, c, dtype=dt) * 0.05).permute(0, 3, 1, 2)
        var, mean = torch.var_mean(x.view(n, h * w, g, c // g).float(), (1, 3), correction=0)
        state["mean"], state["rstd"] = mean, torch.rsqrt(var + EPS)
    if own:
        from paper_2003_06513_gb300 import norm
        state["norm"] = norm
    return state


def _taps(case, shapes, gen):
    """Per weight tensor the taps that each kernel keeps (9 bits), 0 for the kernels pruned away."""
    taps = []
    for shape in shapes:
        if not _masked(shape, case):
            taps.append(None)
            continue
        k = shape[0] * shape[1]
        t = torch.tensor(PATTERNS, dtype=torch.int16)[torch.randint(0, 8, (k,), generator=gen)]
        t[torch.randperm(k, generator=gen)[_kernels_kept(shape, case["keep"]):]] = 0
        taps.append(t.cuda())
    return taps


def _prepare_many(case, seed):
    gen = torch.Generator().manual_seed(seed)
    dev = torch.Generator(device="cuda").manual_seed(seed)
    shapes = _shapes(case["net"])
    sizes = [math.prod(s) for s in shapes]
    taps = _taps(case, shapes, gen)
    spread = [10.0 ** (-4 + 2 * float(r)) for r in torch.rand(len(shapes), generator=gen)]
    grads = [(torch.randn(s, generator=dev, device="cuda") * a).to(DT[case["grad"]]) for s, a in zip(shapes, spread)]
    state = {"case": case, "sizes": sizes, "taps": taps, "grads": grads}
    if case["kind"] == "adamw":
        # the middle of a run: moments and parameters as they are after some steps
        params = [torch.randn(s, generator=dev, device="cuda") * 0.05 for s in shapes]
        keep = _flat_keep(taps, sizes, "cuda")
        scale = torch.cat([torch.full((_padded(k),), a, device="cuda") for k, a in zip(sizes, spread)])
        m = torch.randn(keep.numel(), generator=dev, device="cuda").mul_(scale).mul_(0.3)
        v = torch.rand(keep.numel(), generator=dev, device="cuda").add_(0.5).mul_(scale).mul_(scale)
        m, v = torch.where(keep, m, 0.0), torch.where(keep, v, 0.0)
        _write(params, torch.where(keep, _flat(params), 0.0) if case["keep"] > 0 else _flat(params), sizes)
        state |= {"params": params, "step": 200, "seed": seed & 0x7FFFFFFF,
                  "decay": [DECAY if len(s) == 4 else 0.0 for s in shapes],
                  "grad_scale": torch.rand(1, generator=dev, device="cuda").mul_(0.5).add_(0.5)}
        if case["bits"] == 8:
            r = torch.full((keep.numel(),), 1 << 15, device="cuda")
            state["m"], state["m_scale"] = _encode(m, r, False)
            state["v"], state["v_scale"] = _encode(v, r, True)
        else:
            state["m"], state["v"] = m, v
    if own:
        from paper_2003_06513_gb300 import optim
        if case["kind"] == "adamw":
            held = {k: state[k] for k in ("m", "v", "m_scale", "v_scale", "step") if k in state}
            state["opt"] = optim.AdamW(state["params"], LR, (B1, B2), ADAM_EPS, state["decay"], state_bits=case["bits"],
                                       taps=taps, grad_dtypes=DT[case["grad"]], seed=state["seed"], state=held)
        else:
            state["norm"] = optim.GradNorm(shapes, DT[case["grad"]], taps)
    return state


# ---------------------------------------------------------------------------------------- a pass

def run(state):
    return {"forward": _forward, "backward": _backward, "adamw": _adamw, "grad_norm": _grad_norm}[state["case"]["kind"]](state)


def _act(z, act):
    return z.clamp_min(0.0) if act == "relu" else z / (1 + torch.exp(-z)) if act == "silu" else z


def _groups(t, case):
    """[n, pixels, groups, channels a group] in 32 bits, of a channels-last tensor."""
    return t.permute(0, 2, 3, 1).reshape(case["n"], -1, case["g"], case["c"] // case["g"]).float()


def _back(t, like):
    n, c, h, w = like.shape
    return t.to(like.dtype).view(n, h, w, c).permute(0, 3, 1, 2)


def _forward(state):
    case, x = state["case"], state["x"]
    if own:
        y, mean, rstd = state["norm"].pp_group_norm(x, case["g"], state["gamma"], state["beta"], EPS, case["act"])
        return {"y": y, "mean": mean, "rstd": rstd}
    t = _groups(x, case)
    mean = t.mean((1, 3), keepdim=True)
    d = t - mean
    rstd = 1 / torch.sqrt((d * d).mean((1, 3), keepdim=True) + EPS)
    affine = (case["g"], case["c"] // case["g"])
    z = d * rstd * state["gamma"].view(affine) + state["beta"].view(affine)
    return {"y": _back(_act(z, case["act"]), x), "mean": mean[:, 0, :, 0], "rstd": rstd[:, 0, :, 0]}


def _backward(state):
    case, x = state["case"], state["x"]
    if own:
        dx, dgamma, dbeta = state["norm"].pp_group_norm_backward(
            state["dy"], x, state["mean"], state["rstd"], case["g"], state["gamma"], state["beta"], case["act"])
        return {"dx": dx, "dgamma": dgamma, "dbeta": dbeta}
    affine = (case["g"], case["c"] // case["g"])
    gamma, rstd = state["gamma"].view(affine), state["rstd"][:, None, :, None]
    xh = (_groups(x, case) - state["mean"][:, None, :, None]) * rstd
    dz = _groups(state["dy"], case)
    if case["act"] != "none":
        z = xh * gamma + state["beta"].view(affine)
        if case["act"] == "relu":
            dz = torch.where(z > 0, dz, 0.0)
        else:
            s = 1 / (1 + torch.exp(-z))
            dz = dz * (s + z * s * (1 - s))
    dgamma, dbeta = (dz * xh).sum((0, 1)).view(-1), dz.sum((0, 1)).view(-1)
    dxh = dz * gamma
    a, b = dxh.mean((1, 3), keepdim=True), (dxh * xh).mean((1, 3), keepdim=True)
    return {"dx": _back(rstd * (dxh - a - xh * b), x), "dgamma": dgamma, "dbeta": dbeta}


def _padded(size):
    return -(-size // BLOCK) * BLOCK


def _filled(parts, fill):
    """One after the other, each filled up to whole blocks from `fill`, in one concatenation."""
    return torch.cat([q for t in parts for q in (t, fill[:_padded(t.numel()) - t.numel()])])


def _flat(tensors):
    """The tensors in 32 bits, one after the other, each filled up with zeros to whole blocks."""
    return _filled([t.reshape(-1) for t in tensors], tensors[0].new_zeros(BLOCK)).float()


def _write(tensors, flat, sizes):
    parts = torch.split(flat, [_padded(k) for k in sizes])
    return [t.copy_(p[:t.numel()].view(t.shape)) for t, p in zip(tensors, parts)]


def _flat_keep(taps, sizes, device):
    """Whether an element is kept (all of an unmasked tensor's; none of the fill)."""
    masked = [t for t in taps if t is not None]
    every = torch.ones(max(sizes), dtype=torch.bool, device=device)
    bits = iter(())
    if masked:
        bit = torch.arange(9, device=device, dtype=torch.int16)
        bits = iter(torch.split(((torch.cat(masked)[:, None] >> bit) & 1).bool().view(-1), [9 * t.numel() for t in masked]))
    parts = [every[:k] if t is None else next(bits) for t, k in zip(taps, sizes)]
    return _filled(parts, torch.zeros(BLOCK, dtype=torch.bool, device=device))


# The dither of the 8-bit states: 16 bits for m and 16 for v, from the step's key and the element's
# position (8 consecutive elements share a hash, each multiplies it by its own odd constant: the
# first 32 bits of the fractions of the square roots of the first eight primes, made odd).
ODD = [0x6A09E667, 0xBB67AE85, 0x3C6EF373, 0xA54FF53B, 0x510E527F, 0x9B05688D, 0x1F83D9AB, 0x5BE0CD19]
PHI, WORD = 0x9E3779B1, 0xFFFFFFFF


def _hash(x):
    """A 32-bit mix (its factors: as ODD, of the next two primes), on an int or on int64 values below 2^32."""
    x = x ^ (x >> 16)
    x = (x * 0xCBBB9D5D) & WORD
    x = x ^ (x >> 15)
    x = (x * 0x629A292B) & WORD
    return x ^ (x >> 16)


def _key(seed, step):
    return _hash((seed + step * PHI) & WORD)


def _dither(key, count, device):
    h = _hash(((torch.arange(count // 8, device=device) * PHI) & WORD) ^ key)
    y = (h[:, None] * torch.tensor(ODD, device=device)) & WORD
    y = (y ^ (y >> 15)).view(-1)
    return y & 0xFFFF, y >> 16


def _encode(t, r, positive):
    """8-bit floats (e4m3) and a power of two a block: the block's largest finite value comes to lie
    in (224, 448].  Magnitudes are rounded to one of their two neighbours by the 16-bit dither r; what
    is not finite becomes NaN; a second moment above zero stays above zero."""
    t = t.view(-1, BLOCK)
    a = t.abs()
    fine = a < math.inf
    mant, expo = torch.frexp(torch.where(fine, a, 0.0).amax(1, keepdim=True))
    expo = torch.where(mant > 0, (expo - 9 + (mant > 0.875)).clamp_min(-126), 0)
    scale = torch.ldexp(torch.ones_like(mant), expo)
    a = a * (1 / scale)
    small = torch.where(a < 2.0 ** -6, 2.0 ** -6, 0.0)       # below: the grid of the values just above
    w = (((a + small).view(torch.int32) + ((2 * r.view(-1, BLOCK) + 1) << 3).int()) & ~0xFFFFF).view(torch.float32) - small
    if positive:
        w = torch.where(a > 0, w.clamp_min(2.0 ** -9), w)
    code = torch.where(fine, torch.copysign(w, t), math.nan).to(torch.float8_e4m3fn)
    return code.view(-1), scale.view(-1)


def _decode(code, scale):
    return (code.float().view(-1, BLOCK) * scale[:, None]).view(-1)


def _adamw(state):
    case = state["case"]
    if own:
        state["opt"].step(state["grads"], grad_scale=state["grad_scale"])
    else:
        state["step"] += 1
        t, sizes, eight = state["step"], state["sizes"], case["bits"] == 8
        keep = _flat_keep(state["taps"], sizes, "cuda")
        g, p = _flat(state["grads"]) * state["grad_scale"], _flat(state["params"])
        m = _decode(state["m"], state["m_scale"]) if eight else state["m"]
        v = _decode(state["v"], state["v_scale"]) if eight else state["v"]
        shrink = torch.tensor([1 - LR * d for d in state["decay"]], device="cuda")
        shrink = torch.cat([shrink[i:i + 1].expand(_padded(k)) for i, k in enumerate(sizes)])
        m2 = torch.where(keep, m * B1 + g * (1 - B1), m)
        v2 = torch.where(keep, v * B2 + (g * g) * (1 - B2), v)
        u = (m2 / (1 - B1 ** t)) / (torch.sqrt(v2 / (1 - B2 ** t)) + ADAM_EPS)
        _write(state["params"], torch.where(keep, p * shrink - LR * u, p), sizes)
        if eight:
            rm, rv = _dither(_key(state["seed"], t), m2.numel(), "cuda")
            for name, new, r, positive in (("m", m2, rm, False), ("v", v2, rv, True)):
                code, scale = _encode(new, r, positive)
                state[name].copy_(code)
                state[name + "_scale"].copy_(scale)
        else:
            state["m"].copy_(m2)
            state["v"].copy_(v2)
    return {k: state[k] for k in ("params", "m", "v", "m_scale", "v_scale") if k in state}


def _grad_norm(state):
    if own:
        norm, scale = state["norm"](state["grads"], 1.0)
    else:
        g = torch.where(_flat_keep(state["taps"], state["sizes"], "cuda"), _flat(state["grads"]), 0.0)
        norm = torch.sqrt((g * g).sum()).view(1)
        scale = torch.clamp_max(1.0 / (norm + 1e-6), 1.0)
    return {"norm": norm, "scale": scale}


def work(case):
    """Each input once and each output once; of masked tensors the kept elements and the tap masks."""
    if "act" in case:
        values = case["n"] * case["c"] * case["h"] * case["w"]
        stats, affine = 8 * case["n"] * case["g"], 8 * case["c"]
        if case["kind"] == "forward":
            return {"bytes": 2 * SIZE[case["dtype"]] * values + stats + affine, "flops": (9 + 4 * (case["act"] == "silu")) * values}
        return {"bytes": 3 * SIZE[case["dtype"]] * values + stats + 2 * affine, "flops": (16 + 10 * (case["act"] == "silu")) * values}
    nbytes = flops = 0
    for shape in _shapes(case["net"]):
        size = math.prod(shape)
        kept = 4 * _kernels_kept(shape, case["keep"]) if _masked(shape, case) else size
        nbytes += kept * SIZE[case["grad"]] + (2 * shape[0] * shape[1] if _masked(shape, case) else 0)
        if case["kind"] == "adamw":
            nbytes += kept * (8 + (16 if case["bits"] == 32 else 4)) + (16 * _padded(size) // BLOCK if case["bits"] == 8 else 0)
        flops += kept * (2 if case["kind"] == "grad_norm" else 16 if case["bits"] == 32 else 40)
    return {"bytes": nbytes, "flops": flops}


# ------------------------------------------------------------------- the same in 64 bits

def exact(case, seed):
    state = prepare(case, seed)
    return {"forward": _exact_forward, "backward": _exact_backward, "adamw": _exact_adamw,
            "grad_norm": _exact_norm}[case["kind"]](case, state)


def _exact_forward(case, s):
    n, c, h, w = s["x"].shape
    out, means, rstds = [], [], []
    for i in range(n):
        x = s["x"][i].double().reshape(case["g"], -1)
        mean = x.mean(1)
        rstd = (x.var(1, unbiased=False) + EPS).rsqrt()
        z = ((x - mean[:, None]) * rstd[:, None]).reshape(c, -1) * s["gamma"].double()[:, None] + s["beta"].double()[:, None]
        out.append((z.relu() if case["act"] == "relu" else z * z.sigmoid() if case["act"] == "silu" else z).reshape(c, h, w))
        means.append(mean)
        rstds.append(rstd)
    return {"y": torch.stack(out), "mean": torch.stack(means), "rstd": torch.stack(rstds)}


def _exact_backward(case, s):
    n, c, h, w = s["x"].shape
    per = c // case["g"]
    gamma, beta = s["gamma"].double()[:, None], s["beta"].double()[:, None]
    dgamma = torch.zeros(c, dtype=torch.float64, device="cuda")
    dbeta, dx = torch.zeros_like(dgamma), []
    for i in range(n):
        mean, rstd = (s[k][i].double().repeat_interleave(per)[:, None] for k in ("mean", "rstd"))
        xh = (s["x"][i].double().reshape(c, -1) - mean) * rstd
        z = gamma * xh + beta
        slope = (z > 0).double() if case["act"] == "relu" else torch.ones_like(z)
        if case["act"] == "silu":
            slope = z.sigmoid() * (1 + z * (1 - z.sigmoid()))
        dz = s["dy"][i].double().reshape(c, -1) * slope
        dgamma += (dz * xh).sum(1)
        dbeta += dz.sum(1)
        e = (gamma * dz).reshape(case["g"], -1)
        q = xh.reshape(case["g"], -1)
        d = e - e.mean(1, keepdim=True) - q * (e * q).mean(1, keepdim=True)
        dx.append((d.reshape(c, -1) * rstd).reshape(c, h, w))
    return {"dx": torch.stack(dx), "dgamma": dgamma, "dbeta": dbeta}


def _kept_of(taps, size):
    """Kept elements of one tensor, from its taps, as 0 and 1."""
    if taps is None:
        return torch.ones(size, dtype=torch.float64, device="cuda")
    return torch.stack([(taps.int() // 2 ** t) % 2 for t in range(9)], 1).reshape(-1).double()


def _exact_codes(t, r, floor):
    """The 8-bit form of one tensor's states in 64 bits: (codes, scales)."""
    b = t.view(-1, BLOCK)
    largest = b.abs().amax(1, keepdim=True)
    expo = torch.floor(torch.log2(torch.where(largest > 0, largest, 1.0)))
    expo = torch.where(largest > 1.75 * 2.0 ** expo, expo + 1, expo)
    scale = torch.where(largest > 0, 2.0 ** torch.clamp(expo - 8, min=-126), 1.0)
    a = b.abs() / scale
    step = 2.0 ** (torch.floor(torch.log2(torch.clamp(a, min=2.0 ** -6))) - 3)
    w = torch.floor(a / step + (r.view(-1, BLOCK) + 0.5) / 65536) * step
    w = torch.where(a > 0, torch.clamp(w, min=2.0 ** -9), w) if floor else w
    return (w * torch.sign(b)).view(-1), scale.view(-1)


def _exact_adamw(case, s):
    t, eight = s["step"] + 1, case["bits"] == 8
    got = {k: [] for k in ("params", "m", "v") + (("m_scale", "v_scale") if eight else ())}
    rm, rv = _dither(_key(s["seed"], t), s["m"].numel(), "cuda") if eight else (None, None)
    at = 0
    for p, g, taps, wd in zip(s["params"], s["grads"], s["taps"], s["decay"]):
        size, end = p.numel(), at + _padded(p.numel())
        m, v = s["m"][at:end].double(), s["v"][at:end].double()
        if eight:
            m = m * s["m_scale"][at // BLOCK:end // BLOCK].double().repeat_interleave(BLOCK)
            v = v * s["v_scale"][at // BLOCK:end // BLOCK].double().repeat_interleave(BLOCK)
        k = _kept_of(taps, size)
        g = g.double().reshape(-1) * s["grad_scale"].double() * k
        m[:size] += k * (1 - B1) * (g - m[:size])
        v[:size] += k * (1 - B2) * (g * g - v[:size])
        u = (m[:size] / (1 - B1 ** t)) / ((v[:size] / (1 - B2 ** t)).sqrt() + ADAM_EPS)
        p = p.double().reshape(-1)
        got["params"].append((p - k * LR * (wd * p + u)).view(s["params"][len(got["params"])].shape))
        if eight:
            m, ms = _exact_codes(m, rm[at:end], False)
            v, vs = _exact_codes(v, rv[at:end], True)
            got["m_scale"].append(ms)
            got["v_scale"].append(vs)
        got["m"].append(m)
        got["v"].append(v)
        at = end
    return {k: x if k == "params" else torch.cat(x) for k, x in got.items()}


def _exact_norm(case, s):
    total = torch.zeros(1, dtype=torch.float64, device="cuda")
    for g, taps, size in zip(s["grads"], s["taps"], s["sizes"]):
        total += (g.double().reshape(-1) * _kept_of(taps, size)).square().sum()
    norm = total.sqrt()
    return {"norm": norm, "scale": torch.clamp(1 / (norm + 1e-6), max=1.0)}

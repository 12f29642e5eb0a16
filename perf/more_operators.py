"""What is measured: the operators of distilled retraining of a residual pattern-pruned network.

The pruned network goes back to its user, who retrains it beside the dense network that it came from.
Of that teacher's scores a row's largest logits are kept, and the student is trained on them and on the
labels; in networks with residual blocks a block's output joins the stream through its norm, gate and
scale, and the stream's norm with its activation is what the next block reads.

* ``top``: of each row of logits the k largest (ties to the lowest index), their places, and the
  log-sum-exp of the others at a temperature: what is stored of a teacher.
* ``distill``: loss of a row = (1 - alpha) (log-sum-exp of s - s_label) + alpha T^2 KL(p || q): p the
  softmax of the teacher's kept logits over T, with the others' log-sum-exp as one more class where it is
  given, q the student's softmax over T of the same classes.  A row without a label (below 0) has no
  label's part, one without a kept logit (places below 0) no teacher's.  A training program keeps five
  numbers a row for the backward pass: the largest logit m, the sum of exp(s - m) (0 without labels), the
  sum of exp((s - m) / T), and the last two of the classes that are not kept, the largest and the sum.
* ``distill_back``: the logits' gradient from the rows' gradients.  A row of gradient 0 gets zeros.
  ``distill_step``: both, by the differentiable operation.
* ``block``: h = x + scale_c gate_nc norm(b), y = act(norm(h)); a norm is over a pixel's channels, with
  or without the mean, times a weight and plus a bias a channel; the second one is of h as it is stored.
* ``block_back``: from the gradients of h and y those of x, b and all parameters.

Sizes are those of this repository's networks (10 and 1000 classes; VGG-16, ResNet-50, MobileNet-V2
layers), wide classifiers, and odd sizes between them.
"""
from __future__ import annotations

import math

import torch

own = False

DT = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
SIZE = {"f32": 4, "f16": 2, "bf16": 2}
EPS = 1e-5
LARGEST_BYTES = 2 ** 31     # of a drawn case


# --------------------------------------------------------------------------------------- cases

def _rows(name, kind, rows, classes, k, dtype, t, alpha=0.5, labels=True, rest=True, extra=0):
    case = {"name": name, "kind": kind, "rows": rows, "classes": classes, "k": k, "dtype": dtype, "t": t, "extra": extra}
    return case if kind == "top" else case | {"alpha": alpha, "labels": labels, "rest": rest}


def _block(name, kind, n, c, h, w, dtype, stream, post, pre, act, gate=True, scale=True, bias=True):
    return {"name": name, "kind": kind, "n": n, "c": c, "h": h, "w": w, "dtype": dtype, "stream": stream, "post": post,
            "pre": pre, "act": act, "gate": gate, "scale": scale, "bias": bias}


def listed():
    return [
        # a batch of the teacher's scores of a thousand classes
        _rows("top_1000_n256", "top", 256, 1000, 16, "f32", 2.0),
        # a wide classifier's scores, one step's rows
        _rows("top_32768_r4096_bf16", "top", 4096, 32768, 64, "bf16", 2.0),
        # few rows, very many classes, many kept
        _rows("top_200001_r6", "top", 6, 200001, 200, "f32", 1.0),
        # the small retraining command: ten classes, launch and latency
        _rows("distill_10_n64", "distill", 64, 10, 4, "f32", 2.0, 0.7),
        # as one differentiable call with its backward pass, ragged: an odd row length, rows of a wider tensor,
        # the teacher's kept classes alone
        _rows("distill_step_21841_r1000_f16", "distill_step", 1000, 21841, 50, "f16", 4.0, 0.9, rest=False, extra=3),
        # a wide classifier's step: both parts, the others as a class of their own
        _rows("distill_32768_r8192_bf16", "distill", 8192, 32768, 64, "bf16", 2.0),
        # an ordinary batch of a thousand classes
        _rows("distill_back_1000_n512", "distill_back", 512, 1000, 16, "f32", 2.0),
        # the wide classifier's gradient, the largest case
        _rows("distill_back_65536_r8192_bf16", "distill_back", 8192, 65536, 64, "bf16", 2.0),
        # one small sample in fp32: launch and latency
        _block("block_32_n1", "block", 1, 64, 32, 32, "f32", "f32", "rms", "rms", "relu"),
        # the middle of a residual network in half precision, ordinary batch
        _block("block_56_n32_f16", "block", 32, 256, 56, 56, "f16", "f16", "layer", "layer", "relu"),
        # ragged: odd channels and map, the stream in fp32 beside bf16 blocks
        _block("block_back_ragged", "block_back", 5, 150, 45, 61, "bf16", "f32", "rms", "rms", "silu"),
        # the second stage's gradient in half precision
        _block("block_back_112_n32_f16", "block_back", 32, 128, 112, 112, "f16", "f16", "layer", "layer", "relu"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    while True:
        dtype = rng.choice(["f32", "f16", "bf16"])
        if rng.random() < 0.55:
            rows, classes = _log(rng, 1, 16384), _log(rng, 4, 262144)
            kind = rng.choice(["top", "distill", "distill_back", "distill_step"])
            case = _rows("", kind, rows, classes, _log(rng, 1, min(classes, 256)), dtype,
                         rng.choice([1.0, 1.0, 2.0, 3.0, 4.0]), rng.choice([0.3, 0.5, 0.9, 1.0]), rng.random() < 0.7,
                         rng.random() < 0.6, rng.choice([0, 0, 1, 8]))
        else:
            h = _log(rng, 1, 224)
            w = h if rng.random() < 0.5 else max(1, min(224, int(h * rng.uniform(0.6, 1.6))))
            c = _log(rng, 4, 2048)
            case = _block("", rng.choice(["block", "block_back"]), _log(rng, 1, 64), c // 8 * 8 if c > 8 and rng.random() < 0.6 else c,
                          h, w, dtype, "f32" if rng.random() < 0.25 else dtype, rng.choice(["none", "rms", "layer"]),
                          rng.choice(["rms", "layer", "layer", "none"]), rng.choice(["none", "relu", "silu"]), rng.random() < 0.5,
                          rng.random() < 0.7, rng.random() < 0.7)
            if case["pre"] == "none":
                case["act"] = "none"
        del case["name"]
        if work(case)["bytes"] <= LARGEST_BYTES:
            return case


# ------------------------------------------------------------------------------------ the inputs

def prepare(case, seed):
    state = _prepare_block(case, seed) if "act" in case else _prepare_rows(case, seed)
    if own:
        from paper_2003_06513_gb300 import distill, norm
        state["module"] = norm if "act" in case else distill
    return state


def _prepare_rows(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    r, v, k, dt = case["rows"], case["classes"], case["k"], DT[case["dtype"]]

    def uniform(*shape):
        return torch.rand(*shape, generator=gen, device="cuda")

    # scores: a spread of its own for each row, a few classes well above the others
    wide = torch.randn(r, v + case["extra"], generator=gen, device="cuda", dtype=dt)
    s = wide.mul_((1 + 1.5 * uniform(r, 1)).to(dt))[:, :v]
    # distinct places: the j-th lies in [j v / k, (j + 1) v / k)
    low = (torch.arange(k + 1, device="cuda") * v + k - 1) // k
    width = low[1:] - low[:-1]
    places = low[:-1] + torch.minimum((uniform(r, k) * width).long(), width - 1)
    places = places.gather(1, uniform(r, k).argsort(1))
    top = torch.sort(torch.randn(r, k, generator=gen, device="cuda") * 1.5 + 7, 1, descending=True)[0]
    s.scatter_(1, places, (s.gather(1, places).float() + top * uniform(r, 1)).to(dt))
    state = {"case": case, "s": s}
    if case["kind"] == "top":
        return state
    empty = uniform(r) < 0.05                  # rows that the teacher says nothing about
    state["values"] = top.to(dt)
    state["indices"] = torch.where(empty[:, None], -1, places).int()
    state["rest"] = None
    if case["rest"]:
        state["rest"] = torch.where(empty | (k == v), -math.inf, math.log(max(1, v - k)) + 2 * uniform(r) / case["t"])
    state["labels"] = None
    if case["labels"]:                         # half of them the teacher's first class, a tenth none
        y = torch.where(uniform(r) < 0.5, places[:, 0], torch.randint(0, v, (r,), generator=gen, device="cuda"))
        state["labels"] = torch.where(uniform(r) < 0.1, -100, y)
    if case["kind"] in ("distill_back", "distill_step"):
        state["dloss"] = torch.where(uniform(r) < 0.02, 0.0, (64.0 / r) * (0.5 + uniform(r)))
    if case["kind"] == "distill_back":
        rows = max(1, 2 ** 26 // v)            # the forward pass's five numbers a row
        state["stats"] = torch.cat([_stats(case, state, slice(i, i + rows))[0] for i in range(0, r, rows)])
    return state


def _prepare_block(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    n, c, h, w = case["n"], case["c"], case["h"], case["w"]

    def normal(*shape, dtype=torch.float32):
        return torch.randn(*shape, generator=gen, device="cuda", dtype=dtype)

    def image(dt, spread, shift=0.0):          # every channel with its own spread and shift
        x = normal(n, h, w, c, dtype=DT[dt]).mul_((spread * (0.5 + normal(c).abs())).to(DT[dt]))
        return (x.add_((shift * normal(c)).to(DT[dt])) if shift else x).permute(0, 3, 1, 2)

    def channel(mean, spread, wanted=True):
        return mean + spread * normal(c) if wanted else None

    state = {"case": case, "b": image(case["dtype"], 1.0, 0.3),
             "post_weight": channel(1, 0.1, case["post"] != "none"), "post_bias": channel(0, 0.1, case["post"] != "none" and case["bias"]),
             "weight": channel(1, 0.1, case["pre"] != "none"), "bias": channel(0, 0.1, case["pre"] != "none" and case["bias"]),
             "scale": channel(0.2, 0.05, case["scale"]), "gate": torch.sigmoid(normal(n, c)) if case["gate"] else None}
    state["x" if case["kind"] == "block" else "h"] = image(case["stream"], 1.5, 0.5)
    if case["kind"] == "block_back":
        state["dh"] = image(case["stream"], 0.05)
        state["dy"] = image(case["dtype"], 0.05) if case["pre"] != "none" else None
    return state


# ---------------------------------------------------------------------------------------- a pass

def run(state):
    return {"top": _top, "distill": _distill, "distill_back": _distill_back, "distill_step": _distill_step, "block": _forward,
            "block_back": _backward}[state["case"]["kind"]](state)


def _top(state):
    case, s = state["case"], state["s"]
    if own:
        values, indices, rest = state["module"].pp_top_logits(s, case["k"], case["t"])
        return {"values": values, "indices": indices, "rest": rest}
    x, order = torch.sort(s, dim=1, descending=True, stable=True)
    k = case["k"]
    if k < case["classes"]:
        others = x[:, k:].float()
        rest = others[:, 0] / case["t"] + torch.log(torch.exp((others - others[:, :1]) / case["t"]).sum(1))
    else:
        rest = torch.full((case["rows"],), -math.inf, device="cuda")
    return {"values": x[:, :k].contiguous(), "indices": order[:, :k].int(), "rest": rest}


def _teacher(case, state, rows):
    """(p of the kept classes, of the others, the places, which of them there are, whether a row has any): p in 32 bits."""
    places = state["indices"][rows].long()
    there = (places >= 0) & (places < case["classes"])
    t = torch.where(there, state["values"][rows].float() / case["t"], -math.inf)
    if state["rest"] is not None:
        t = torch.cat([t, state["rest"][rows, None]], 1)
    top = t.amax(1, keepdim=True)
    some = top[:, 0] > -math.inf
    e = torch.exp(t - torch.where(some[:, None], top, 0.0))
    p = e / torch.where(some[:, None], e.sum(1, keepdim=True), 1.0)
    log_p = t - torch.where(some[:, None], top + torch.log(e.sum(1, keepdim=True)), 0.0)
    return p, log_p, places, there, some


def _stats(case, state, rows):
    """(the five numbers a row, the logits in 32 bits, the classes that are not kept, the teacher's side)"""
    s = state["s"][rows].float()
    teacher = p, log_p, places, there, some = _teacher(case, state, rows)
    others = torch.ones(s.shape[0], case["classes"] + 1, dtype=torch.bool, device="cuda")
    if state["rest"] is not None:
        others.scatter_(1, torch.where(there, places, case["classes"]), False)
    others = others[:, :case["classes"]]
    m = s.amax(1, keepdim=True)
    z1 = torch.exp(s - m).sum(1) if state["labels"] is not None else torch.zeros_like(m[:, 0])
    zt = torch.exp((s - m) / case["t"]).sum(1)
    o = torch.where(others, s, -math.inf)
    mo = o.amax(1, keepdim=True)
    zo = torch.exp((o - torch.where(mo > -math.inf, mo, 0.0)) / case["t"]).sum(1)
    stats = torch.stack([m[:, 0], z1, zt, mo[:, 0], zo], 1)
    if state["labels"] is not None:
        some = some | (state["labels"][rows] >= 0)
    return torch.where(some[:, None], stats, 0.0), s, others, teacher


def _distill(state):
    case, alpha, t, everything = state["case"], state["case"]["alpha"], state["case"]["t"], slice(None)
    if own:
        loss, stats = state["module"].pp_distill(state["s"], state["values"], state["indices"], state["rest"], state["labels"], t, alpha)
        return {"loss": loss, "stats": stats}
    stats, s, others, (p, log_p, places, there, some) = _stats(case, state, everything)
    m, z1, zt, mo, zo = stats.unbind(1)
    log_q = (s.gather(1, torch.where(there, places, 0)) - m[:, None]) / t - torch.log(zt)[:, None]
    if state["rest"] is not None:
        log_q = torch.cat([log_q, ((mo - m) / t + torch.log(zo) - torch.log(zt))[:, None]], 1)
    loss = torch.where(some, alpha * t * t * torch.where(p > 0, p * (log_p - log_q), 0.0).sum(1), 0.0)
    if state["labels"] is not None:
        y = state["labels"]
        own_score = s.gather(1, y.clamp_min(0)[:, None])[:, 0]
        loss = loss + torch.where(y >= 0, (1 - alpha) * (torch.log(z1) - (own_score - m)), 0.0)
    return {"loss": loss, "stats": stats}


def _distill_back(state):
    t, alpha = state["case"]["t"], state["case"]["alpha"]
    if own:
        return {"ds": state["module"].pp_distill_backward(state["dloss"], state["s"], state["stats"], state["values"], state["indices"],
                                                          state["rest"], state["labels"], t, alpha)}
    return {"ds": _slopes(state, state["stats"])}


def _distill_step(state):
    case = state["case"]
    if own:
        s = state["s"].detach().requires_grad_(True)
        module = state["module"]
        top = module.TopLogits(state["values"], state["indices"], state["rest"])
        loss = module.distill_loss(s, top, state["labels"], case["t"], case["alpha"])
        return {"loss": loss.detach(), "ds": torch.autograd.grad(loss, s, state["dloss"])[0]}
    forward = _distill(state)
    return {"loss": forward["loss"], "ds": _slopes(state, forward["stats"])}


def _slopes(state, stats):
    case, alpha, t = state["case"], state["case"]["alpha"], state["case"]["t"]
    p, _, places, there, some = _teacher(case, state, slice(None))
    s, k = state["s"].float(), case["k"]
    m, z1, zt, mo, zo = (c[:, None] for c in stats.unbind(1))
    ds = torch.exp((s - mo) / t) / zo
    if state["rest"] is not None:
        ds = ds * (torch.exp((mo - m) / t) * zo / zt - p[:, k:])
        column = torch.where(there, places, case["classes"])
        kept = torch.exp((s.gather(1, torch.where(there, places, 0)) - m) / t) / zt - p[:, :k]
        ds = torch.cat([ds, ds[:, :1]], 1).scatter_(1, column, kept)[:, :case["classes"]]
    else:
        ds = ds.scatter_add_(1, torch.where(there, places, 0), torch.where(there, -p, 0.0))
    ds = torch.where(some[:, None], alpha * t * ds, 0.0)
    if state["labels"] is not None:
        y = state["labels"][:, None]
        q = (torch.exp(s - m) / z1).scatter_add_(1, y.clamp_min(0), torch.full_like(m, -1.0))
        ds = ds + torch.where(y >= 0, (1 - alpha) * q, 0.0)
    g = state["dloss"][:, None]
    return torch.where(g == 0, 0.0, ds * g).to(state["s"].dtype)


def _last(t):
    """[n, pixels, channels] in 32 bits of a channels-last tensor."""
    return t.permute(0, 2, 3, 1).flatten(1, 2).float()


def _back(t, like, dtype):
    n, c, h, w = like.shape
    return t.to(dtype).view(n, h, w, c).permute(0, 3, 1, 2)


def _hat(t, kind):
    """(the normalised values, 1 / root): over the last dimension, without its mean where it is a layer norm."""
    if kind == "none":
        return t, None
    d = t - t.mean(2, keepdim=True) if kind == "layer" else t
    r = 1 / torch.sqrt((d * d).mean(2, keepdim=True) + EPS)
    return d * r, r


def _affine(t, weight, bias):
    t = t if weight is None else t * weight
    return t if bias is None else t + bias


def _unhat(d, hat, r, kind):
    """The gradient of what was normalised, from that of the normalised values."""
    if kind == "none":
        return d
    a = d.mean(2, keepdim=True) if kind == "layer" else 0.0
    return r * (d - a - hat * (d * hat).mean(2, keepdim=True))


def _arguments(state):
    case = state["case"]
    return dict(post=case["post"], post_weight=state["post_weight"], post_bias=state["post_bias"], scale=state["scale"],
                gate=state["gate"], pre=case["pre"], weight=state["weight"], bias=state["bias"], act=case["act"], eps=EPS)


def _forward(state):
    case, x, b = state["case"], state["x"], state["b"]
    if own:
        h, y = state["module"].pp_block_norm(x, b, **_arguments(state))
        return {"h": h} if y is None else {"h": h, "y": y}
    u = _affine(_hat(_last(b), case["post"])[0], state["post_weight"], state["post_bias"])
    u = u if state["scale"] is None else u * state["scale"]
    u = u if state["gate"] is None else u * state["gate"][:, None]
    h = _back(_last(x) + u, x, x.dtype)
    if case["pre"] == "none":
        return {"h": h}
    z = _affine(_hat(_last(h), case["pre"])[0], state["weight"], state["bias"])
    z = z.clamp_min(0.0) if case["act"] == "relu" else z / (1 + torch.exp(-z)) if case["act"] == "silu" else z
    return {"h": h, "y": _back(z, x, b.dtype)}


def _backward(state):
    case, h, b = state["case"], state["h"], state["b"]
    if own:
        got = state["module"].pp_block_norm_backward(state["dh"], state["dy"], h, b, **_arguments(state))
        return {k: t for k, t in got._asdict().items() if t is not None}
    out, dh = {}, _last(state["dh"])
    if case["pre"] != "none":
        hat, r = _hat(_last(h), case["pre"])
        dz = _last(state["dy"])
        if case["act"] == "relu":              # on which side of the kink z lies takes 64 bits
            z = _affine(_hat(_last(h).double(), case["pre"])[0], state["weight"].double(), state["bias"])
            dz = torch.where(z > 0, dz, 0.0)
        elif case["act"] == "silu":
            z = _affine(hat, state["weight"], state["bias"])
            sig = 1 / (1 + torch.exp(-z))
            dz = dz * (sig + z * sig * (1 - sig))
        out["dweight"] = (dz * hat).sum((0, 1))
        if state["bias"] is not None:
            out["dbias"] = dz.sum((0, 1))
        dh = dh + _unhat(dz * state["weight"], hat, r, case["pre"])
    out["dx"] = _back(dh, h, h.dtype)
    hat, r = _hat(_last(b), case["post"])
    u = _affine(hat, state["post_weight"], state["post_bias"])
    du, one = dh, torch.ones(1, device="cuda")
    scale, gate = (one if state[k] is None else state[k] for k in ("scale", "gate"))
    joined = (dh * u).sum(1)
    if state["gate"] is not None:
        out["dgate"] = scale * joined
        gate = gate[:, None]
    if state["scale"] is not None:
        out["dscale"] = (gate.flatten(1) * joined if state["gate"] is not None else joined).sum(0)
    du = dh * scale * gate
    if case["post"] != "none":
        out["dpost_weight"] = (du * hat).sum((0, 1))
        if state["post_bias"] is not None:
            out["dpost_bias"] = du.sum((0, 1))
        du = du * state["post_weight"]
    out["dblock"] = _back(_unhat(du, hat, r, case["post"]), b, b.dtype)
    return {k: out[k] for k in ("dx", "dblock", "dpost_weight", "dpost_bias", "dscale", "dgate", "dweight", "dbias") if k in out}


def work(case):
    """Each input once and each output once."""
    if "act" in case:
        values, c = case["n"] * case["h"] * case["w"] * case["c"], case["c"]
        a, s, pre = SIZE[case["dtype"]], SIZE[case["stream"]], case["pre"] != "none"
        vectors = 4 * c * (2 * (case["post"] != "none") + 2 * pre + case["scale"] + case["n"] * case["gate"])
        if case["kind"] == "block":
            return {"bytes": values * (2 * s + a * (1 + pre)) + vectors, "flops": values * (8 + 8 * pre + 4 * (case["act"] == "silu"))}
        return {"bytes": values * (3 * s + a * (2 + pre)) + 2 * vectors, "flops": values * (16 + 16 * pre + 8 * (case["act"] == "silu"))}
    values, es, r, k = case["rows"] * case["classes"], SIZE[case["dtype"]], case["rows"], case["k"]
    if case["kind"] == "top":
        return {"bytes": values * es + r * (k * (es + 4) + 4), "flops": 4 * values}
    teacher = r * (k * (es + 4) + 4 * case["rest"] + 8 * case["labels"])
    both = case["labels"] and case["t"] != 1
    if case["kind"] == "distill":
        return {"bytes": values * es + teacher + 24 * r, "flops": values * (4 + 3 * both)}
    # (a step reads its logits again for the gradient: nothing keeps them between the two calls)
    step = case["kind"] == "distill_step"
    return {"bytes": (2 + step) * values * es + teacher + 24 * r, "flops": values * (5 + 4 * both + step * (4 + 3 * both))}


# ------------------------------------------------------------------- the same in 64 bits

def exact(case, seed):
    state = prepare(case, seed)
    return {"top": _exact_top, "block": _exact_block, "block_back": _exact_block_back}.get(case["kind"], _exact_distill)(case, state)


def _pieces(case, most=2 ** 25):
    step = max(1, most // case["classes"])
    return [slice(i, min(case["rows"], i + step)) for i in range(0, case["rows"], step)]


def _exact_top(case, state):
    got = {"values": [], "indices": [], "rest": []}
    for rows in _pieces(case):
        s = state["s"][rows].double()
        at = torch.sort(-s, dim=1, stable=True)[1][:, :case["k"]]
        got["values"].append(s.gather(1, at))
        got["indices"].append(at.int())
        got["rest"].append(torch.logsumexp(s.scatter(1, at, -math.inf) / case["t"], 1))
    return {k: torch.cat(v) for k, v in got.items()}


def _exact_distill(case, state):
    """Both directions: the loss and the five numbers, or its derivative by every logit."""
    t, alpha, v, kind = case["t"], case["alpha"], case["classes"], case["kind"]
    losses, numbers, slopes = [], [], []
    for rows in _pieces(case):
        s = state["s"][rows].double()
        r = s.shape[0]
        at = state["indices"][rows].long()
        given = at >= 0
        at = at.clamp_min(0)
        log_t = torch.where(given, state["values"][rows].double() / t, -math.inf)
        log_qall = torch.log_softmax(s / t, 1)
        mask = torch.zeros_like(s)
        if case["rest"]:
            mask.scatter_(1, at, given.double())
            log_t = torch.cat([log_t, state["rest"][rows, None].double()], 1)
        left = torch.where(mask > 0, -math.inf, s)
        has = (log_t > -math.inf).any(1)
        log_p = log_t - torch.where(has, torch.logsumexp(log_t, 1), 0.0)[:, None]
        p = torch.where(has[:, None], log_p.exp(), 0.0)
        log_left = torch.logsumexp(torch.where(mask > 0, -math.inf, log_qall), 1)
        log_q = log_qall.gather(1, at)
        if case["rest"]:
            log_q = torch.cat([log_q, log_left[:, None]], 1)
        y = state["labels"][rows] if case["labels"] else torch.full((r,), -1, device="cuda")
        if kind != "distill":
            d = torch.where(has[:, None], log_qall.exp(), 0.0)
            d.scatter_add_(1, at, torch.where(given, -p[:, :case["k"]], 0.0))
            if case["rest"]:
                inside = torch.exp(torch.where(mask > 0, -math.inf, log_qall) - torch.where(log_left > -math.inf, log_left, 0.0)[:, None])
                d -= p[:, -1:] * inside
            hard = torch.softmax(s, 1).scatter_add_(1, y.clamp_min(0)[:, None], torch.full((r, 1), -1.0, dtype=s.dtype, device="cuda"))
            d = alpha * t * d + torch.where(y >= 0, 1 - alpha, 0.0)[:, None] * hard
            slopes.append(d * state["dloss"][rows, None].double())
        if kind == "distill_back":
            continue
        kl = torch.where(p > 0, p * (log_p - log_q), 0.0).sum(1)
        ce = -torch.log_softmax(s, 1).gather(1, y.clamp_min(0)[:, None])[:, 0]
        losses.append(alpha * t * t * kl + torch.where(y >= 0, (1 - alpha) * ce, 0.0))
        m, mo = s.amax(1), left.amax(1)
        shift = torch.where(mo > -math.inf, mo, 0.0)
        five = [m, torch.exp(s - m[:, None]).sum(1) * case["labels"], torch.exp((s - m[:, None]) / t).sum(1), mo,
                torch.exp((left - shift[:, None]) / t).sum(1)]
        numbers.append(torch.stack(five, 1) * 1.0)
        numbers[-1][~(has | (y >= 0))] = 0.0
    if kind == "distill_back":
        return {"ds": torch.cat(slopes)}
    return {"loss": torch.cat(losses)} | ({"stats": torch.cat(numbers)} if kind == "distill" else {"ds": torch.cat(slopes)})


def _sample(t, i):
    return t[i].double().flatten(1)                       # [channels, pixels]


def _column(t):
    return None if t is None else t.double()[:, None]


def _normed(v, kind, weight, bias):
    """(weight xh + bias, xh, the function that takes a gradient of xh back to v) of one sample."""
    if kind == "none":
        return v, v, lambda g: g
    centre = v.mean(0) if kind == "layer" else torch.zeros_like(v[0])
    root = torch.sqrt(((v - centre) ** 2).mean(0) + EPS)
    xh = (v - centre) / root

    def back(g):
        g = (g - xh * (g * xh).mean(0)) / root
        return g - g.mean(0) if kind == "layer" else g
    z = xh if weight is None else xh * _column(weight)
    return z if bias is None else z + _column(bias), xh, back


def _factor(case, state, i):
    f = torch.ones(case["c"], 1, dtype=torch.float64, device="cuda")
    f = f if state["scale"] is None else f * _column(state["scale"])
    return f if state["gate"] is None else f * _column(state["gate"][i])


def _exact_block(case, state):
    hs, ys = [], []
    for i in range(case["n"]):
        u = _normed(_sample(state["b"], i), case["post"], state["post_weight"], state["post_bias"])[0]
        h = _sample(state["x"], i) + _factor(case, state, i) * u
        hs.append(h.view(state["x"].shape[1:]))
        z = _normed(h.to(state["x"].dtype).double(), case["pre"], state["weight"], state["bias"])[0]
        z = z.relu() if case["act"] == "relu" else z * z.sigmoid() if case["act"] == "silu" else z
        ys.append(z.view(state["x"].shape[1:]))
    return {"h": torch.stack(hs)} if case["pre"] == "none" else {"h": torch.stack(hs), "y": torch.stack(ys)}


def _exact_block_back(case, state):
    c, zero = case["c"], torch.zeros(case["c"], dtype=torch.float64, device="cuda")
    one = torch.ones(c, 1, dtype=torch.float64, device="cuda")
    got = {k: zero.clone() for k in ("dpost_weight", "dpost_bias", "dscale", "dweight", "dbias")}
    dxs, dbs, dgates = [], [], []
    for i in range(case["n"]):
        d = _sample(state["dh"], i)
        if case["pre"] != "none":
            z, xh, back = _normed(_sample(state["h"], i), case["pre"], state["weight"], state["bias"])
            dz = _sample(state["dy"], i)
            if case["act"] == "relu":
                dz = dz * (z > 0)
            elif case["act"] == "silu":
                dz = dz * z.sigmoid() * (1 + z * (1 - z.sigmoid()))
            got["dweight"] += (dz * xh).sum(1)
            got["dbias"] += dz.sum(1)
            d = d + back(dz * _column(state["weight"]))
        dxs.append(d.view(state["h"].shape[1:]))
        u, bh, back = _normed(_sample(state["b"], i), case["post"], state["post_weight"], state["post_bias"])
        scale = one if state["scale"] is None else _column(state["scale"])
        gate = one if state["gate"] is None else _column(state["gate"][i])
        dgates.append((d * u * scale).sum(1))
        got["dscale"] += (d * u * gate).sum(1)
        du = d * scale * gate
        got["dpost_weight"] += (du * bh).sum(1)
        got["dpost_bias"] += du.sum(1)
        dbs.append(back(du if state["post_weight"] is None else du * _column(state["post_weight"])).view(state["b"].shape[1:]))
    got |= {"dx": torch.stack(dxs), "dblock": torch.stack(dbs), "dgate": torch.stack(dgates)}
    there = {"dx": True, "dblock": True, "dpost_weight": case["post"] != "none", "dpost_bias": state["post_bias"] is not None,
             "dscale": case["scale"], "dgate": case["gate"], "dweight": case["pre"] != "none", "dbias": state["bias"] is not None}
    return {k: got[k] for k, wanted in there.items() if wanted}

"""A teacher's top logits, the distillation loss with its gradient, and block norm, in plain float64 numpy.

TEST INFRASTRUCTURE ONLY (see the package docstring).  It pins pp_top_logits, pp_distill, pp_distill_backward, pp_block_norm
and pp_block_norm_backward (include/patconv.h); the *_bound results sum the first-order effects of fp32 roundings, so that
a tolerance follows from the inputs and not from a trial.
"""
from __future__ import annotations

import numpy as np

from .train import act, slope

U = 2.0 ** -24      # half a unit in the last place of fp32


def _lse(x, axis=1):
    """log-sum-exp; -inf of nothing."""
    m = x.max(axis, keepdims=True) if x.shape[axis] else np.full(x.shape[:axis] + (1,) + x.shape[axis + 1:], -np.inf)
    shift = np.where(np.isfinite(m), m, 0.0)
    with np.errstate(divide="ignore"):
        return (np.log(np.exp(x - shift).sum(axis, keepdims=True)) + shift).squeeze(axis)


# ------------------------------------------------------------------------------------- top logits

def top(s, k, t):
    """(values, indices, rest) of each row, by a stable sort of the row in falling order, NaN first."""
    s = np.asarray(s, np.float64)
    key = np.where(np.isnan(s), np.inf, s)
    order = np.lexsort((np.broadcast_to(np.arange(s.shape[1]), s.shape), -key, ~np.isnan(s)), axis=1)
    ranked = np.take_along_axis(s, order, 1)
    return ranked[:, :k], order[:, :k], _lse(ranked[:, k:] / t)


# ------------------------------------------------------------------------------------- distillation

def _teacher(values, indices, rest, classes, t):
    """Masses of the classes [rows, classes] and, last, of the others; entropy term sum p log p a row; rows that have any."""
    values, indices = np.asarray(values, np.float64), np.asarray(indices, np.int64)
    there = (indices >= 0) & (indices < classes)
    u = np.where(there, values / t, -np.inf)
    if rest is not None:
        u = np.concatenate([u, np.asarray(rest, np.float64)[:, None]], 1)
    some = (u > -np.inf).any(1)
    lse = np.where(some, _lse(u), 0.0)
    log_p = u - lse[:, None]
    p = np.where(some[:, None], np.exp(log_p), 0.0)
    return p, log_p, there, some


def distill(s, values, indices, rest, labels, t, alpha):
    """(loss, stats, gradient by the logits for a loss gradient of 1, sizes of the terms of the losses, of the gradients):
    an fp32 result is off by a number of roundings (``roundings``) of the terms' sizes."""
    s = np.asarray(s, np.float64)
    rows, classes = s.shape
    p, log_p, there, some = _teacher(values, indices, rest, classes, t)
    k = indices.shape[1]
    at = np.where(there, indices, 0)
    m = s.max(1)
    far = (s - np.where(np.isfinite(m), m, 0.0)[:, None]) / t       # (s / t by itself may be so large that 64 bits lose the sum's log beside it)
    log_q = far - _lse(far)[:, None]
    kept = np.zeros((rows, classes), bool)
    for j in range(k):
        kept[np.arange(rows)[there[:, j]], at[there[:, j], j]] = True
    o = np.where(kept, -np.inf, s) if rest is not None else s
    mo = o.max(1)
    zo = np.exp((o - np.where(np.isfinite(mo), mo, 0.0)[:, None]) / t).sum(1)
    q = np.take_along_axis(log_q, at, 1)
    log_q0 = _lse(np.where(kept, -np.inf, log_q))
    if rest is not None:
        q = np.concatenate([q, log_q0[:, None]], 1)
    with np.errstate(invalid="ignore"):
        terms = np.where(p > 0, p * (log_p - q), 0.0)
    loss = np.where(some, alpha * t * t * terms.sum(1), 0.0) if alpha else np.zeros(rows)      # (no weight takes no part, an infinite one neither)
    # gradient: alpha T (q_v - p_v), where a class of the others has its share of q_0 - p_0
    grad = np.exp(log_q)
    reach = grad.copy()
    if rest is not None:
        with np.errstate(invalid="ignore"):
            inside = np.where(zo[:, None] > 0, np.exp((o - mo[:, None]) / t) / np.where(zo > 0, zo, 1.0)[:, None], 0.0)
        grad = np.where(kept, grad, (np.exp(log_q0) - p[:, k])[:, None] * inside)
        reach = np.where(kept, reach, (np.exp(log_q0) + p[:, k])[:, None] * inside)
    for j in range(k):
        r = np.nonzero(there[:, j])[0]
        np.add.at(grad, (r, at[r, j]), -p[r, j])
        np.add.at(reach, (r, at[r, j]), p[r, j])
    grad, reach = (alpha * t * np.where(some[:, None], g, 0.0) for g in (grad, reach))
    with np.errstate(invalid="ignore"):
        parts = np.where(p > 0, p * (np.abs(log_p) + np.abs(q) + 1), 0).sum(1)
    largest = np.where(there & np.isfinite(values), np.abs(values), 0.0).max(1)
    size = np.abs(loss) + alpha * t * largest + (alpha * t * t * parts if alpha else 0.0)
    z1 = np.zeros(rows)
    useful = some.copy()
    if labels is not None:
        y = np.asarray(labels, np.int64)
        has = (y >= 0) & (y < classes)
        useful |= has
        z1 = np.exp(s - m[:, None]).sum(1)
        yy = np.where(has, y, 0)
        ce = np.log(z1) - (s[np.arange(rows), yy] - m)
        if alpha < 1:
            loss = loss + np.where(has, (1 - alpha) * ce, 0.0)
        if alpha < 1:
            size = size + np.where(has, (1 - alpha) * (np.abs(np.log(z1)) + np.abs(s[np.arange(rows), yy] - m) + 1), 0.0)
        hard = np.exp(s - m[:, None]) / z1[:, None]
        reach = reach + np.where(has[:, None], (1 - alpha) * hard, 0.0)
        hard[np.arange(rows), yy] -= 1
        reach[np.arange(rows), yy] += np.where(has, 1 - alpha, 0.0)
        grad = grad + np.where(has[:, None], (1 - alpha) * hard, 0.0)
    zt = np.exp((s - m[:, None]) / t).sum(1)
    stats = np.stack([m, z1, zt, mo, zo], 1)
    stats[~useful] = 0
    # the exponents are rounded too: that counts for more the further a logit is below the largest
    reach = reach * (1 + np.where(np.isfinite(s), m[:, None] - s, 0.0) / (32 * min(t, 1.0)))
    return loss, stats, grad, size, reach


def roundings(classes):
    """Roundings, relative to the terms' sizes, that a result may be off by: 64 for exponentials, factors and joins, and those
    of a thread's running sum, which takes a 64th of a short row (a warp's, in pairs) or a 512th of a long one."""
    return U * (64 + (classes / 64 if classes <= 2048 else classes / 512))


# ------------------------------------------------------------------------------------- block norm

def _hat(v, kind, eps):
    """(v^, 1 / root): over the channels, the last dimension."""
    if kind == "none":
        return v, np.ones(v.shape[:-1] + (1,))
    d = v - v.mean(-1, keepdims=True) if kind == "layer" else v
    with np.errstate(divide="ignore", invalid="ignore"):
        r = 1 / np.sqrt((d * d).mean(-1, keepdims=True) + eps)
    return d * r, r


def _or(p, value):
    return value if p is None else np.asarray(p, np.float64)


def _rows(t):
    """[N, pixels, C] of [N, C, H, W]."""
    n, c = t.shape[:2]
    return np.moveaxis(np.asarray(t, np.float64).reshape(n, c, -1), 1, 2)


def _image(t, like):
    return np.moveaxis(t, 2, 1).reshape(like.shape)


E = 2.0 ** -19      # 32 fp32 roundings, as for the group norm


def _hat_error(v, hat, r, kind):
    """Of v^ in fp32.  Its own roundings and the root's are relative to |v^|.  A layer norm's mean is the sum of C distances from a
    value near it, over C: the sum's 3 + 5 + 4 levels of additions (a thread's eight values, a warp, sixteen warps) round by
    2^-24 of the distances' mean size each, which is at most 1 / r (the root of their mean square) and the near value's own distance,
    at most that again for values in no special order; times r that is 12 * 2 * 2^-24 < E, whatever |v^|.  And values far from
    zero hold their distances to 2^-24 of the mean's size alone, which E / 8 of it covers four times."""
    if kind == "none":
        return 0 * hat
    return E * (np.abs(hat) + ((1 + np.abs(v.mean(-1, keepdims=True)) * r * 2.0 ** -3) if kind == "layer" else 0.0))


def block_h(x, b, post, pw, pb, scale, gate, eps):
    """(h before it is rounded, bound of its fp32 error): x + scale gate (pw b^ + pb)."""
    v = _rows(b)
    hat, r = _hat(v, post, eps)
    f = _or(scale, 1.0) * (1.0 if gate is None else np.asarray(gate, np.float64)[:, None])
    u = _or(pw, 1.0) * hat + _or(pb, 0.0)
    bound = np.abs(f) * (np.abs(_or(pw, 1.0)) * (_hat_error(v, hat, r, post) + E * np.abs(hat)) + E * np.abs(_or(pb, 0.0))) + U * 4 * np.abs(_rows(x))
    return _image(_rows(x) + f * u, x), _image(bound + 0 * hat, x)


def block_y(h, pre, w, bias, kind, eps):
    """(y, bound) from h as it is stored."""
    v = _rows(h)
    hat, r = _hat(v, pre, eps)
    z = _or(w, 1.0) * hat + _or(bias, 0.0)
    y = act(z, kind)
    bound = 1.1 * (np.abs(_or(w, 1.0)) * _hat_error(v, hat, r, pre) + E * np.abs(_or(bias, 0.0))) + E * np.abs(y)
    return _image(y, h), _image(bound, h)


def block_backward(dh, dy, h, b, post, pw, pb, scale, gate, pre, w, bias, kind, eps):
    """Gradients and their fp32 bounds, as two dicts; every parameter's, whether it is there or not."""
    n = h.shape[0]
    zeros = np.zeros_like(_rows(h))
    d = zeros if dh is None else _rows(dh)
    d_e = U * np.abs(d)
    out, bound = {}, {}

    def through(g, g_e, hat, hat_e, r, layer):
        """The gradient of v from that of v^, with the errors of both."""
        a = g.mean(-1, keepdims=True) if layer else 0.0
        a_e = g_e.mean(-1, keepdims=True) + E * np.abs(g).mean(-1, keepdims=True) if layer else 0.0
        c = (g * hat).mean(-1, keepdims=True)
        c_e = (g_e * np.abs(hat) + np.abs(g) * hat_e + E * np.abs(g * hat)).mean(-1, keepdims=True)
        full = r * (g - a - hat * c)
        e = r * (g_e + a_e + np.abs(hat) * c_e + hat_e * np.abs(c) + E * (np.abs(g) + np.abs(a) + np.abs(hat * c)))
        return full, e

    if dy is not None and pre != "none":
        v = _rows(h)
        hat, r = _hat(v, pre, eps)
        hat_e = _hat_error(v, hat, r, pre)
        z = _or(w, 1.0) * hat + _or(bias, 0.0)
        g = _rows(dy)
        dz = g * slope(z, kind)
        z_e = np.abs(_or(w, 1.0)) * hat_e + E * (np.abs(z) + np.abs(_or(bias, 0.0)))
        dz_e = np.abs(g) * (0.5 * z_e + E) if kind == "silu" else U * np.abs(dz)      # which side of the kink: in 64 bits
        out["dweight"], out["dbias"] = (dz * hat).sum((0, 1)), dz.sum((0, 1))
        bound["dweight"] = (dz_e * np.abs(hat) + np.abs(dz) * hat_e + E * np.abs(dz * hat)).sum((0, 1))
        bound["dbias"] = (dz_e + E * np.abs(dz)).sum((0, 1))
        t = dz * _or(w, 1.0)
        full, e = through(t, np.abs(_or(w, 1.0)) * dz_e + U * np.abs(t), hat, hat_e, r, pre == "layer")
        d, d_e = d + full, d_e + e + U * np.abs(d + full)
    out["dx"], bound["dx"] = _image(d, h), _image(d_e, h)
    if b is None:
        return out, bound
    v = _rows(b)
    hat, r = _hat(v, post, eps)
    hat_e = _hat_error(v, hat, r, post)
    sc = _or(scale, 1.0) * np.ones(h.shape[1])
    ga = np.ones((n, h.shape[1])) if gate is None else np.asarray(gate, np.float64)
    pwv, pbv = _or(pw, 1.0) * np.ones(h.shape[1]), _or(pb, 0.0) * np.ones(h.shape[1])
    e, f = (d * hat).sum(1), d.sum(1)
    e_e = (d_e * np.abs(hat) + np.abs(d) * hat_e + E * np.abs(d * hat)).sum(1)
    f_e = (d_e + E * np.abs(d)).sum(1)
    joined, j_e = pwv * e + pbv * f, np.abs(pwv) * e_e + np.abs(pbv) * f_e
    out["dgate"], bound["dgate"] = sc * joined, np.abs(sc) * (j_e + E * np.abs(joined))
    out["dscale"], bound["dscale"] = (ga * joined).sum(0), (np.abs(ga) * (j_e + E * np.abs(joined))).sum(0)
    out["dpost_weight"], bound["dpost_weight"] = (sc * ga * e).sum(0), (np.abs(sc * ga) * (e_e + E * np.abs(e))).sum(0)
    out["dpost_bias"], bound["dpost_bias"] = (sc * ga * f).sum(0), (np.abs(sc * ga) * (f_e + E * np.abs(f))).sum(0)
    k = (sc * ga * pwv)[:, None]
    t, t_e = d * k, d_e * np.abs(k) + 4 * U * np.abs(d * k)
    if post != "none":
        t, t_e = through(t, t_e, hat, hat_e, r, post == "layer")
    out["dblock"], bound["dblock"] = _image(t, h), _image(t_e, h)
    return out, bound

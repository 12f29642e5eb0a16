"""Group norm with its activation, the gradients' norm and AdamW steps in plain float64 numpy.

TEST INFRASTRUCTURE ONLY (see the package docstring).  It pins the operators of masked retraining
(include/patconv.h: pp_group_norm, pp_grad_norm, pp_adamw_step) and says how far fp32 arithmetic may be
from them: the *_bound functions sum the first-order effects of roundings of relative size ``e`` on
every intermediate value, so that a tolerance follows from the inputs and not from a trial.
"""
from __future__ import annotations

import numpy as np

E = 2.0 ** -19      # 32 fp32 roundings: the products, the sums' joins, and exp's own error (about 2 + |z| ulp)


# ------------------------------------------------------------------------------------- group norm

def act(z, kind):
    if kind == "relu":
        return np.where(np.isnan(z), z, np.maximum(z, 0.0))
    if kind == "silu":
        with np.errstate(over="ignore", invalid="ignore"):
            return z / (1.0 + np.exp(-z))
    return z


def slope(z, kind):
    if kind == "relu":
        return (z > 0).astype(np.float64)
    if kind == "silu":
        with np.errstate(over="ignore"):
            s = 1.0 / (1.0 + np.exp(-z))
        return s + z * s * (1 - s)
    return np.ones_like(z)


def _grouped(t, groups):
    """[N, C, ...] as [N, G, C / G, pixels]."""
    n, c = t.shape[:2]
    return np.asarray(t, np.float64).reshape(n, groups, c // groups, -1)


def _channel(p, groups, default, c):
    p = np.full(c, default) if p is None else np.asarray(p, np.float64)
    return p.reshape(1, groups, c // groups, 1)


def norm_forward(x, groups, gamma, beta, eps, kind):
    """(y, mean, rstd, bound of y's fp32 error before its rounding to the output type)."""
    g = _grouped(x, groups)
    c = x.shape[1]
    mean = g.mean((2, 3), keepdims=True)
    rstd = 1.0 / np.sqrt(((g - mean) ** 2).mean((2, 3), keepdims=True) + eps)
    xh = (g - mean) * rstd
    ga, be = _channel(gamma, groups, 1.0, c), _channel(beta, groups, 0.0, c)
    z = ga * xh + be
    y = act(z, kind)
    # xh is off by roundings of x - mean and of rstd, and by the mean's error, which its sum of |x| sets;
    # |act'| <= 1.1
    spread = np.abs(g).mean((2, 3), keepdims=True) * rstd
    bound = 1.1 * E * (np.abs(ga) * (np.abs(xh) + spread) + np.abs(be)) + E * np.abs(y)
    return y.reshape(x.shape), mean[:, :, 0, 0], rstd[:, :, 0, 0], bound.reshape(x.shape)


def norm_backward(dy, x, mean, rstd, groups, gamma, beta, kind):
    """((dx, dgamma, dbeta), bounds of their fp32 errors); mean and rstd as given."""
    c = x.shape[1]
    mu, r = (np.asarray(t, np.float64).reshape(x.shape[0], groups, 1, 1) for t in (mean, rstd))
    g, d = _grouped(x, groups), _grouped(dy, groups)
    ga, be = _channel(gamma, groups, 1.0, c), _channel(beta, groups, 0.0, c)
    xh = (g - mu) * r
    z = ga * xh + be
    dz = d * slope(z, kind)
    e = ga * dz
    a, b = e.mean((2, 3), keepdims=True), (e * xh).mean((2, 3), keepdims=True)
    dx = r * (e - a - xh * b)
    dgamma, dbeta = (dz * xh).sum((0, 3)).reshape(c), dz.sum((0, 3)).reshape(c)
    # first-order bounds: xh_e, z_e, dz_e are the absolute errors of xh, z and dz
    xh_e = E * (np.abs(xh) + np.abs(mu) * r)
    z_e = np.abs(ga) * xh_e + E * (np.abs(z) + np.abs(be))
    if kind == "relu":                    # a slope that rounding may have turned over
        dz_e = np.where(np.abs(z) <= z_e, np.abs(d), 0.0)
    else:
        dz_e = np.abs(d) * (0.5 * z_e + E) if kind == "silu" else np.zeros_like(d)     # |silu''| <= 0.5
    e_e = np.abs(ga) * dz_e + E * np.abs(e)
    a_e = e_e.mean((2, 3), keepdims=True)
    exh_e = e_e * np.abs(xh) + np.abs(e) * xh_e + E * np.abs(e * xh)
    b_e = exh_e.mean((2, 3), keepdims=True)
    dx_e = r * (e_e + a_e + E * np.abs(a) + np.abs(xh) * b_e + np.abs(b) * (xh_e + E * np.abs(xh))) + E * np.abs(dx)
    dgamma_e = (dz_e * np.abs(xh) + np.abs(dz) * xh_e + E * np.abs(dz * xh)).sum((0, 3)).reshape(c)
    dbeta_e = (dz_e + E * np.abs(dz)).sum((0, 3)).reshape(c)
    return (dx.reshape(x.shape), dgamma, dbeta), (dx_e.reshape(x.shape), dgamma_e, dbeta_e)


# ------------------------------------------------------------------------------------- many tensors

def kept(taps, numel):
    """Whether each element is kept: all without masks, else bit t of its nine's mask for raster tap t."""
    if taps is None:
        return np.ones(numel, bool)
    return ((np.asarray(taps, np.int64)[:, None] >> np.arange(9)) & 1).astype(bool).reshape(-1)


def grad_norm(grads, taps, max_norm):
    total = 0.0
    for g, t in zip(grads, taps):
        if g is not None:
            g = np.asarray(g, np.float64).reshape(-1)
            total += float((g[kept(t, g.size)] ** 2).sum())
    norm = np.sqrt(total)
    return norm, min(1.0, max_norm / (norm + 1e-6))


def adamw(p, g, m, v, taps, lr, b1, b2, eps, decay, step):
    """New (p, m, v) of one tensor, flat, in 64 bits; elements left out keep theirs."""
    k = kept(taps, p.size)
    m2, v2 = b1 * m + (1 - b1) * g, b2 * v + (1 - b2) * g * g
    with np.errstate(invalid="ignore", divide="ignore"):
        u = (m2 / (1 - b1 ** step)) / (np.sqrt(v2 / (1 - b2 ** step)) + eps)
    p2 = p * (1 - lr * decay) - lr * u
    return np.where(k, p2, p), np.where(k, m2, m), np.where(k, v2, v)


# ------------------------------------------------------------------------------------- 8-bit states

BLOCK = 256
_M = 0xFFFFFFFF
# odd parts of the first 32 bits of the fractions of the square roots of the primes 2 to 29
_ROOTS = [(int(np.floor((np.sqrt(np.longdouble(q)) % 1) * 2 ** 32)) & _M) | 1 for q in (2, 3, 5, 7, 11, 13, 17, 19, 23, 29)]
_PHI = 0x9E3779B1


def _mix(x):
    x = np.asarray(x, np.uint64) & np.uint64(_M)
    x ^= x >> np.uint64(16)
    x = (x * np.uint64(_ROOTS[8])) & np.uint64(_M)
    x ^= x >> np.uint64(15)
    x = (x * np.uint64(_ROOTS[9])) & np.uint64(_M)
    return x ^ (x >> np.uint64(16))


def dither(seed, step, first, count):
    """16 bits for m and 16 for v of elements first .. first + count - 1 of the states (multiples of 8)."""
    key = _mix((seed + step * _PHI) & _M)
    eights = np.arange(first // 8, (first + count) // 8, dtype=np.uint64)
    h = _mix(((eights * np.uint64(_PHI)) & np.uint64(_M)) ^ key)
    y = (h[:, None] * np.array(_ROOTS[:8], np.uint64)) & np.uint64(_M)
    y = (y ^ (y >> np.uint64(15))).reshape(-1)
    return (y & np.uint64(0xFFFF)).astype(np.int64), (y >> np.uint64(16)).astype(np.int64)


def encode(t, r, positive):
    """(values over the scale, scale per element, margin): the 8-bit form of whole blocks, flat.  The
    margin is how far the position between two neighbours was from where the rounding turns, in steps."""
    b = np.asarray(t, np.float64).reshape(-1, BLOCK)
    a = np.abs(b)
    fine = np.isfinite(a)
    top = np.where(fine, a, 0.0).max(1, keepdims=True)
    mant, expo = np.frexp(top)                             # mant in [0.5, 1)
    scale = np.where(top > 0, 2.0 ** np.maximum(expo - 9 + (mant > 0.875), -126), 1.0)
    a = np.where(fine, a / scale, 0.0)
    step = 2.0 ** (np.floor(np.log2(np.maximum(a, 2.0 ** -6))) - 3)
    at = a / step + (r.reshape(-1, BLOCK) + 0.5) / 65536
    w = np.floor(at) * step
    if positive:
        w = np.where(a > 0, np.maximum(w, 2.0 ** -9), w)
    w = np.where(fine, np.copysign(w, b), np.nan)
    return w.reshape(-1), np.broadcast_to(scale, b.shape).reshape(-1), np.abs(at - np.round(at)).reshape(-1)

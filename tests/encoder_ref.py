"""Plain references of the encoder operators in 64 bits (numpy, CPU), token by token
or as the formulas stand, and bounds on the error that a kernel may have.

A bound is elementwise: the result's own rounding (unit roundoff of its type), plus
what sums in float may lose (their length times 2^-23 of the sum of magnitudes),
plus, where a kernel's operands are rounded on the way, that roundoff of the sum of
magnitudes.  The sums of magnitudes are the same formulas on absolute values.
"""
import numpy as np

UNIT = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}
F32 = 2.0 ** -23
# what rounding to a subnormal may lose at least
TINY = {"f32": 2.0 ** -149, "bf16": 2.0 ** -133, "f16": 2.0 ** -24}


def norm(x, w, b, eps):
    mean = x.mean(1)
    var = ((x - mean[:, None]) ** 2).mean(1)
    rstd = 1.0 / np.sqrt(var + eps)
    y = (x - mean[:, None]) * rstd[:, None]
    if w is not None:
        y = y * w
    return (y if b is None else y + b), mean, rstd


def norm_grad(dy, x, w, mean, rstd):
    xh = (x - mean[:, None]) * rstd[:, None]
    g = dy if w is None else dy * w
    dx = rstd[:, None] * (g - g.mean(1, keepdims=True) - xh * (g * xh).mean(1, keepdims=True))
    return dx, (dy * xh).sum(0), dy.sum(0)


def attention(q, k, v, g, scale, bounds, s0=None):
    """q [n, H, dk], k, v [n, Hk, d], sequences bounds[i]..bounds[i+1]: o, final states; the recurrence."""
    n, H, dk = q.shape
    Hk, dv = v.shape[1:]
    c = np.arange(H) // (H // Hk)
    lam = np.exp(g)[:, None, None]
    o = np.zeros((n, H, dv))
    last = np.zeros((len(bounds) - 1, H, dk, dv))
    for s in range(len(bounds) - 1):
        S = np.zeros((H, dk, dv)) if s0 is None else s0[s].copy()
        for t in range(bounds[s], bounds[s + 1]):
            S = lam * S + k[t][c][:, :, None] * v[t][c][:, None, :]
            o[t] = scale * np.einsum("hi,hij->hj", q[t], S)
        last[s] = S
    return o, last


def attention_grad(do, q, k, v, g, scale, bounds, s0=None, ds=None):
    """dq, dk, dv, d s0 by the reverse recurrence."""
    n, H, dk_ = q.shape
    Hk, dv_ = v.shape[1:]
    grp = H // Hk
    c = np.arange(H) // grp
    lam = np.exp(g)[:, None, None]
    dq, dk, dv = np.zeros(q.shape), np.zeros(k.shape), np.zeros(v.shape)
    d0 = np.zeros((len(bounds) - 1, H, dk_, dv_))
    for s in range(len(bounds) - 1):
        S = np.zeros((H, dk_, dv_)) if s0 is None else s0[s].copy()
        for t in range(bounds[s], bounds[s + 1]):
            S = lam * S + k[t][c][:, :, None] * v[t][c][:, None, :]
            dq[t] = scale * np.einsum("hij,hj->hi", S, do[t])
        D = np.zeros((H, dk_, dv_)) if ds is None else ds[s].copy()
        for t in range(bounds[s + 1] - 1, bounds[s] - 1, -1):
            D = D + scale * q[t][:, :, None] * do[t][:, None, :]
            dk[t] = np.einsum("hij,hj->hi", D, v[t][c]).reshape(Hk, grp, dk_).sum(1)
            dv[t] = np.einsum("hij,hi->hj", D, k[t][c]).reshape(Hk, grp, dv_).sum(1)
            D = lam * D
        d0[s] = D
    return dq, dk, dv, d0


def _erf(x):
    from math import erf
    return np.vectorize(erf, otypes=[float])(x)


def act(name, g):
    """Value and derivative."""
    with np.errstate(over="ignore"):
        s = 1.0 / (1.0 + np.exp(-g))
    if name == "silu":
        return g * s, s * (1.0 + g * (1.0 - s))
    if name == "gelu":
        p = 0.5 * (1.0 + _erf(g / np.sqrt(2.0)))
        return g * p, p + g * np.exp(-0.5 * g * g) / np.sqrt(2.0 * np.pi)
    if name == "sigmoid":
        return s, s * (1.0 - s)
    return np.maximum(g, 0.0), (g > 0).astype(float)


def ffn(x, wg, wu, name):
    g, u = x @ wg.T, x @ wu.T
    return act(name, g)[0] * u


def ffn_bound(x, wg, wu, name, kind):
    """Bound on |h - exact|: the activations' slope is at most 1.13."""
    g, u = x @ wg.T, x @ wu.T
    ax, n = np.abs(x), x.shape[1] + 8
    eg, eu = n * F32 * (ax @ np.abs(wg).T), n * F32 * (ax @ np.abs(wu).T)
    f = np.abs(act(name, g)[0])
    h = f * np.abs(u)
    e = 1.13 * eg * np.abs(u) + f * eu + 1.13 * eg * eu + 8 * F32 * (1 + np.abs(g)) * h + 4 * F32 * np.abs(u)
    return UNIT[kind] * (h + e) + e + TINY[kind]


def ffn_grad(dh, x, wg, wu, name):
    g, u = x @ wg.T, x @ wu.T
    f, d = act(name, g)
    dg, du = dh * u * d, dh * f
    return dg @ wg + du @ wu, dg.T @ x, du.T @ x


def ffn_grad_bound(dh, x, wg, wu, name, kind):
    """Bounds on the three gradients: those of dg and du (with their rounding as operands; the derivatives' slopes
    are at most 1 / 2, or 0.8 for gelu), carried through the products."""
    g, u = x @ wg.T, x @ wu.T
    ax, n = np.abs(x), x.shape[1] + 8
    eg, eu = n * F32 * (ax @ np.abs(wg).T), n * F32 * (ax @ np.abs(wu).T)
    f, d = act(name, g)
    ah = np.abs(dh)
    dg, du = ah * np.abs(u * d), ah * np.abs(f)
    slope = 0.8
    edg = ah * (eu * (np.abs(d) + slope * eg) + slope * eg * np.abs(u) + 16 * F32 * (1 + np.abs(g)) * np.abs(u))
    edu = ah * (1.13 * eg + 16 * F32 * (1 + np.abs(g)) * (np.abs(f) + 1e-30) + 4 * F32)
    edg = edg + UNIT[kind] * (dg + edg) + TINY[kind]
    edu = edu + UNIT[kind] * (du + edu) + TINY[kind]
    awg, awu = np.abs(wg), np.abs(wu)
    dx, dwg, dwu = (np.abs(t) for t in ffn_grad(dh, x, wg, wu, name))
    m, r = 2 * wg.shape[0] + 64, x.shape[0] + 64
    ex = edg @ awg + edu @ awu + m * F32 * ((dg + edg) @ awg + (du + edu) @ awu)
    ewg = edg.T @ ax + r * F32 * ((dg + edg).T @ ax)
    ewu = edu.T @ ax + r * F32 * ((du + edu).T @ ax)
    return tuple(UNIT[kind] * (v + e) + e + TINY[kind] for v, e in ((dx, ex), (dwg, ewg), (dwu, ewu)))


def attention_bound(parts, kind, tokens, width, whole=False):
    """Bound for an attention result whose value is `parts[0]` and whose sum of magnitudes is `parts[1]`: sums over
    tokens and width, and the pairs' products rounded once as operands (16-bit types).  whole: a state, in float."""
    value, mags = np.abs(parts[0]), np.abs(parts[1])
    e = (2 * tokens + width + 64) * F32 * mags
    if whole:
        return e + 1e-37
    if kind != "f32":
        e = e + UNIT[kind] * mags
    return UNIT[kind] * (value + e) + e + TINY[kind]

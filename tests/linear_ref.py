"""Plain references of the projections in 64 bits (torch, on the tensors' device), and bounds on the error that a kernel
may have: a result's own rounding, and what sums in float may lose (as in encoder_ref)."""
import math

import torch

from encoder_ref import F32, TINY, UNIT

ACTS = [None, "silu", "gelu", "sigmoid", "relu"]


def act(name, z):
    """Value and derivative."""
    if name is None:
        return z, torch.ones_like(z)
    if name == "relu":
        return z.clamp(min=0), (z > 0).double()
    if name == "gelu":
        p = 0.5 * torch.erfc(-z * math.sqrt(0.5))
        return z * p, p + z * torch.exp(-0.5 * z * z) / math.sqrt(2 * math.pi)
    s = torch.sigmoid(z)
    return (s, s * (1 - s)) if name == "sigmoid" else (z * s, s * (1 + z * (1 - s)))


def linear(x, w, b=None, name=None, r=None):
    z = x @ w.T if b is None else x @ w.T + b
    y = act(name, z)[0]
    return y if r is None else y + r


def z_error(x, w, b):
    """On z = x w^T + b in float."""
    mags = x.abs() @ w.abs().T
    return (x.shape[1] + 10) * F32 * (mags if b is None else mags + b.abs())


def linear_bound(x, w, b, name, r, kind):
    """The activations' slopes are at most 1.13; they are formed in a few roundings of values of about 1 + |z|."""
    z = x @ w.T if b is None else x @ w.T + b
    y = act(name, z)[0]
    ez = z_error(x, w, b)
    e = ez if name in (None, "relu") else 1.13 * ez + 8 * F32 * (1 + z.abs()) * (y.abs() + 1e-30)
    out = y.abs() if r is None else (y + r).abs()
    if r is not None:
        e = e + F32 * out
    return UNIT[kind] * (out + e) + e + TINY[kind]


def linear_grad(dy, x, w, b, name):
    z = x @ w.T if b is None else x @ w.T + b
    dz = dy * act(name, z)[1]
    return dz @ w, dz.T @ x, dz.sum(0)


def linear_grad_bounds(dy, x, w, b, name, kind):
    """dz with its rounding as an operand (the derivatives' slopes are at most 0.8; relu's jumps at 0, which z may lie on
    either side of), carried through the products."""
    z = x @ w.T if b is None else x @ w.T + b
    slope = act(name, z)[1]
    dz, edz = (dy * slope).abs(), torch.zeros_like(z)
    if name is not None:
        ez = z_error(x, w, b)
        edz = dy.abs() * (0.8 * ez + 16 * F32 * (1 + z.abs()) if name != "relu" else (z.abs() <= ez).double())
        edz = edz + UNIT[kind] * (dz + edz) + TINY[kind]
    aw, ax, n, rows = w.abs(), x.abs(), w.shape[0], x.shape[0]
    dx, dw, db = (t.abs() for t in linear_grad(dy, x, w, b, name))
    ex = edz @ aw + (n + 80) * F32 * ((dz + edz) @ aw)
    ew = edz.T @ ax + (rows + 80) * F32 * ((dz + edz).T @ ax)
    eb = edz.sum(0) + (rows + 80) * F32 * (dz + edz).sum(0)
    return tuple(UNIT[kind] * (v + e) + e + TINY[kind] for v, e in ((dx, ex), (dw, ew), (db, eb)))

"""Plain references of the root-mean-square norm and of rows in 8 bits, in 64 bits (numpy, CPU), and bounds on the
error that a kernel may have (as in encoder_ref: a result's own rounding, and what sums in float may lose)."""
import numpy as np

from encoder_ref import F32, TINY, UNIT

E4M3 = 2.0 ** -4        # unit roundoff
E4M3_TINY = 2.0 ** -10  # half the step below 2^-6


def rms(h, w, eps):
    rstd = 1.0 / np.sqrt((h ** 2).mean(1) + eps)
    y = h * rstd[:, None]
    return (y if w is None else y * w), rstd


def rms_grad(dy, h, w, rstd, dh=None):
    hh = h * rstd[:, None]
    g = dy if w is None else dy * w
    dx = rstd[:, None] * (g - hh * (g * hh).mean(1, keepdims=True))
    return (dx if dh is None else dx + dh), (dy * hh).sum(0)


def rms_bound(y, n, kind):
    """The sum of squares has no cancellation: off by its length's roundings, half of them in the root."""
    e = (n + 16) * F32 * np.abs(y)
    return UNIT[kind] * (np.abs(y) + e) + e + TINY[kind]


def rms_grad_bounds(dy, h, w, rstd, dh, kind):
    rows, n = h.shape
    hh, g = np.abs(h) * rstd[:, None], np.abs(dy if w is None else dy * w)
    e = (n + 16) * F32 * rstd[:, None] * (g + hh * (g * hh).mean(1, keepdims=True))
    if dh is not None:
        e = e + F32 * np.abs(dh)
    dx, dw = rms_grad(dy, h, w, rstd, dh)
    ew = (rows + 16) * F32 * (np.abs(dy) * hh).sum(0)
    return UNIT[kind] * (np.abs(dx) + e) + e + TINY[kind], UNIT[kind] * (np.abs(dw) + ew) + ew + TINY[kind]


def row_scale(y):
    return np.maximum(np.abs(y).max(1), 448 * 2.0 ** -126) / 448


def rows_8bit_bound(y, scale, e):
    """On |byte * scale - y| for values y that are off by e themselves: half a step of e4m3 (a step is never more
    than twice the roundoff of the value, with what moves it across), and a few roundings in float."""
    return E4M3 * (np.abs(y) + e) + E4M3_TINY * scale[:, None] + e + 8 * F32 * np.abs(y)

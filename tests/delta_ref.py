"""Plain references of attention by the gated delta rule in 64 bits (numpy, CPU), token by token, and bounds on the error
that a kernel may have.

Where |k_t| and beta_t are at most 1, a token's step S -> a (I - beta k^T k) S never lengthens a column of the state: what
a column is off by stays, decayed, and each token adds what its own sums lose.  With W the sum of the decayed |u|-sized
inputs (a bound on a column's length), a token adds at most a few hundred roundings of W + |v|: the products over dk, those
of a chunk's 32 tokens (whose inverse has no entry above 1: it is a product of such steps between two keys), and the
update.  E sums that up.
"""
import numpy as np

from encoder_ref import F32, TINY, UNIT


def heads_of(x, H):
    """q's and k's heads, once for each of v's that read them."""
    return np.repeat(x, H // x.shape[1], axis=1)


def attention(q, k, v, g, beta, scale, bounds, s0=None):
    """q, k [n, Hk, dk], v [n, H, dv], g, beta [n, H], sequences bounds[i]..bounds[i+1]: o, final states, and for each
    token u and the state before it, decayed."""
    n, H, dv = v.shape
    q, k = heads_of(q, H), heads_of(k, H)
    dk = q.shape[2]
    o, u, decayed = np.zeros((n, H, dv)), np.zeros((n, H, dv)), np.zeros((n, H, dk, dv))
    last = np.zeros((len(bounds) - 1, H, dk, dv))
    for s in range(len(bounds) - 1):
        S = np.zeros((H, dk, dv)) if s0 is None else s0[s].copy()
        for t in range(bounds[s], bounds[s + 1]):
            S = np.exp(g[t])[:, None, None] * S
            decayed[t] = S
            u[t] = beta[t][:, None] * (v[t] - np.einsum("hi,hij->hj", k[t], S))
            S = S + k[t][:, :, None] * u[t][:, None, :]
            o[t] = scale * np.einsum("hi,hij->hj", q[t], S)
        last[s] = S
    return o, last, u, decayed


def attention_grad(do, q, k, v, g, beta, scale, bounds, s0=None, ds=None):
    """dq, dk, dv, dg, dbeta, d s0 by the reverse recurrence."""
    n, H, dv_ = v.shape
    Hk = q.shape[1]
    _, _, u, decayed = attention(q, k, v, g, beta, scale, bounds, s0)
    q, k = heads_of(q, H), heads_of(k, H)
    dq, dk, dv, dg, db = np.zeros(q.shape), np.zeros(k.shape), np.zeros(v.shape), np.zeros(g.shape), np.zeros(g.shape)
    d0 = np.zeros((len(bounds) - 1, H, q.shape[2], dv_))
    for s in range(len(bounds) - 1):
        D = np.zeros(d0.shape[1:]) if ds is None else ds[s].copy()
        for t in range(bounds[s + 1] - 1, bounds[s] - 1, -1):
            Sd = decayed[t]
            S = Sd + k[t][:, :, None] * u[t][:, None, :]
            dq[t] = scale * np.einsum("hij,hj->hi", S, do[t])
            D = D + scale * q[t][:, :, None] * do[t][:, None, :]
            du = np.einsum("hi,hij->hj", k[t], D)
            dv[t] = beta[t][:, None] * du
            db[t] = (du * (v[t] - np.einsum("hi,hij->hj", k[t], Sd))).sum(1)
            dk[t] = np.einsum("hij,hj->hi", D, u[t]) - np.einsum("hij,hj->hi", Sd, dv[t])
            D = D - k[t][:, :, None] * dv[t][:, None, :]
            dg[t] = (D * Sd).sum((1, 2))
            D = np.exp(g[t])[:, None, None] * D
        d0[s] = D
    fold = lambda x: x.reshape(n, Hk, H // Hk, -1).sum(2)
    return fold(dq), fold(dk), dv, dg, db, d0


def bounds_forward(q, k, v, g, beta, scale, bounds, s0, o, last, kind):
    n, H, dv = v.shape
    q = heads_of(q, H)
    dk = q.shape[2]
    c = (dk + 1500) * F32
    e_o, e_last = np.zeros(o.shape), np.zeros(last.shape)
    for s in range(len(bounds) - 1):
        W = np.zeros((H, dv)) if s0 is None else np.sqrt((s0[s] ** 2).sum(1))
        E = W.copy()
        for t in range(bounds[s], bounds[s + 1]):
            a, b = np.exp(g[t])[:, None], beta[t][:, None]
            W = a * W + b * np.abs(v[t])
            E = a * E + W + np.abs(v[t])
            qn = np.sqrt((q[t] ** 2).sum(1))[:, None]
            # and what two parts leave out, where the result has 16 bits
            e_o[t] = abs(scale) * qn * (c * E + (0 if kind == "f32" else 2.0 ** -13) * (W + np.abs(v[t])))
        e_last[s] = (c * E)[:, None, :]
    return UNIT[kind] * (np.abs(o) + e_o) + e_o + TINY[kind], e_last + 1e-37


def bounds_grad(do, q, k, v, g, beta, scale, bounds, s0, ds, grads, kind):
    """Bounds on the gradients' errors, from lengths of the columns of S (W), of its gradient (Z) and of what a token writes,
    and what the states are off by (E, F): backwards as forwards, a token adds at most a few hundred roundings of what there is."""
    n, H, dv = v.shape
    Hk, dk = q.shape[1:]
    q = heads_of(q, H)
    c = (dk + 1500) * F32
    qn = np.sqrt((q ** 2).sum(2))[:, :, None]
    do = np.abs(do)
    W, E, Z, F = (np.zeros((n, H, dv)) for _ in range(4))
    d0 = np.zeros((len(bounds) - 1, H, dv))
    for s in range(len(bounds) - 1):
        w = np.zeros((H, dv)) if s0 is None else np.sqrt((s0[s] ** 2).sum(1))
        e = w.copy()
        for t in range(bounds[s], bounds[s + 1]):
            a, b = np.exp(g[t])[:, None], beta[t][:, None]
            w0 = w
            w = a * w + b * np.abs(v[t])
            e = a * e + w + np.abs(v[t])
            W[t], E[t] = np.maximum(w, a * w0) + np.abs(v[t]), e + w
        z = np.zeros((H, dv)) if ds is None else np.sqrt((ds[s] ** 2).sum(1))
        f = z.copy()
        for t in range(bounds[s + 1] - 1, bounds[s] - 1, -1):
            a = np.exp(g[t])[:, None]
            z = z + abs(scale) * qn[t] * do[t]
            f = f + z
            Z[t], F[t] = z, f
            z, f = a * z, a * f
        d0[s] = f
    # what two parts leave out, where the result has 16 bits
    two = 0 if kind == "f32" else 2.0 ** -13
    both = (4 * c * (F * W + Z * E) + two * Z * W).sum(2)
    fold = lambda x: x.reshape(n, Hk, H // Hk).sum(2)[:, :, None]
    of_q = fold((abs(scale) * do * (4 * c * E + two * W)).sum(2))
    # dg adds up what up to 64 tokens pass on
    off = (of_q, fold(2 * both), beta[:, :, None] * (4 * c * F + two * Z), 64 * both, both)
    found = [UNIT[kind] * (np.abs(x) + y) + y + TINY[kind] for x, y in zip(grads, off)]
    return found + [(4 * c * d0)[:, :, None, :] + 1e-37]

"""The encoder operators without a GPU: what the C entry points refuse before
anything is enqueued, workspace sizes, and the references that the GPU tests
compare with, pinned to each other and to differences.
"""
import ctypes

import numpy as np
import pytest

import encoder_ref as ref

nd = pytest.importorskip("paper_2607_03574_amd")
FAKE = 1 << 20      # an address that no refused call reads


def test_norm_refusals():
    ok = dict(dtype=0, x=FAKE, rows=4, n=8, ld_x=8, w=None, b=None, eps=1e-5, y=FAKE, ld_y=8, mean=None, rstd=None)

    def call(**kw):
        return nd._norm(*{**ok, **kw}.values(), None)

    for kw in (dict(dtype=3), dict(dtype=-1), dict(rows=-1), dict(n=0), dict(ld_x=7), dict(ld_y=7), dict(eps=-1.0),
               dict(eps=float("nan")), dict(x=None), dict(y=None), dict(rows=1 << 62, ld_x=1 << 62)):
        assert call(**kw) == nd.E_ARG, kw
        assert "ndvm_layer_norm" in nd.last_error()
    assert call(rows=0, x=None, y=None) == nd.OK


def test_norm_grad_refusals():
    ok = dict(dtype=1, dy=FAKE, ld_dy=8, x=FAKE, ld_x=8, rows=4, n=8, w=None, mean=FAKE, rstd=FAKE, dx=FAKE, ld_dx=8,
              dw=FAKE, db=FAKE, ws=FAKE, bytes=1 << 20)

    def call(**kw):
        return nd._norm_grad(*{**ok, **kw}.values(), None)

    for kw in (dict(dtype=5), dict(mean=None), dict(rstd=None), dict(dy=None), dict(x=None), dict(ld_dx=7), dict(ws=None),
               dict(ws=FAKE + 2)):
        assert call(**kw) == nd.E_ARG, kw
    assert call(bytes=16) == nd.E_NOMEM
    assert call(dx=None, dw=None, db=None, ws=None, bytes=0) == nd.OK       # nothing wanted


def shape(**kw):
    d = dict(dtype=1, n_seq=2, n_tokens=10, heads=4, kv_heads=2, dk=8, dv=16, scale=1.0)
    return nd._AttentionShape(*{**d, **kw}.values())


def heads(data=FAKE, seq=100, tok=10, head=1):
    return nd._Heads(data, seq, tok, head)


def test_attention_refusals():
    def call(s=None, q=None, k=None, v=None, o=None, decay=FAKE, offsets=None, ws=FAKE, bytes=1 << 30):
        return nd._attn(s if s is not None else shape(), q or heads(), k or heads(), v or heads(), decay, offsets, None,
                        o or heads(), None, ws, bytes, None)

    for kw in (dict(dtype=9), dict(n_seq=-1), dict(n_tokens=-1), dict(n_tokens=11), dict(heads=0), dict(heads=3), dict(dk=0),
               dict(dv=-4), dict(scale=float("inf")), dict(n_seq=0)):
        assert call(s=shape(**kw)) == nd.E_ARG, kw
    for kw in (dict(dk=257), dict(dv=300), dict(heads=65536, kv_heads=1), dict(n_tokens=1 << 40, n_seq=1)):
        assert call(s=shape(**kw)) == nd.E_UNSUPPORTED, kw
    for name in "qkvo":
        assert call(**{name: heads(data=None)}) == nd.E_ARG
        assert call(**{name: heads(tok=-1)}) == nd.E_ARG
        assert call(**{name: heads(head=1 << 60)}) == nd.E_ARG
    assert call(decay=None) == nd.E_ARG
    long = shape(n_seq=1, n_tokens=8192)
    assert call(s=long, bytes=0) == nd.E_NOMEM
    assert call(s=long, ws=None) == nd.E_ARG
    assert nd._attn(None, heads(), heads(), heads(), FAKE, None, None, heads(), None, None, 0, None) == nd.E_ARG


def test_attention_grad_and_step_refusals():
    s = shape()
    n = nd._sz()
    assert nd._attn_ws(s, 0, 1, ctypes.byref(n)) == nd.OK and n.value > 0
    none = nd._Heads(None, 0, 0, 0)

    def grad(do=None, dv=None, d0=None, ws=FAKE, bytes=n.value):
        return nd._attn_grad(s, heads(), heads(), heads(), FAKE, None, None, do or heads(), None, heads(), heads(),
                             dv or heads(), d0, ws, bytes, None)

    assert grad(do=none) == nd.E_ARG
    assert grad(dv=none, d0=FAKE) == nd.E_ARG
    assert grad(ws=None) == nd.E_ARG
    assert grad(bytes=n.value - 1) == nd.E_NOMEM

    def step(s=s, slots=FAKE, n_slots=4, state=FAKE, q=None):
        return nd._attn_step(s, q or heads(), heads(), heads(), FAKE, state, n_slots, slots, heads(), None)

    assert step(slots=None, n_slots=1) == nd.E_ARG
    assert step(state=None) == nd.E_ARG
    assert step(n_slots=-1) == nd.E_ARG
    assert step(q=none) == nd.E_ARG
    assert step(s=shape(dk=1000)) == nd.E_UNSUPPORTED
    assert step(s=shape(n_seq=0)) == nd.OK


def test_ffn_refusals():
    # (few rows need no workspace)
    ok = dict(dtype=1, act=0, x=FAKE, rows=400, n_in=8, ld_x=8, wg=FAKE, ld_g=8, wu=FAKE, ld_u=8, n_out=16, h=FAKE, ld_h=16, ws=FAKE,
              bytes=1 << 30)

    def call(**kw):
        return nd._ffn(*{**ok, **kw}.values(), None)

    for kw in (dict(dtype=7), dict(act=4), dict(act=-1), dict(rows=-1), dict(n_in=0), dict(n_out=0), dict(ld_x=7), dict(ld_g=7),
               dict(ld_u=7), dict(ld_h=15), dict(x=None), dict(wg=None), dict(wu=None), dict(h=None), dict(ws=None)):
        assert call(**kw) == nd.E_ARG, kw
    for kw in (dict(rows=1 << 23), dict(n_in=1 << 22, ld_x=1 << 22, ld_g=1 << 22, ld_u=1 << 22), dict(n_out=1 << 22, ld_h=1 << 22)):
        assert call(**kw) == nd.E_UNSUPPORTED, kw
    assert call(bytes=10) == nd.E_NOMEM
    assert call(rows=0, x=None, h=None) == nd.OK
    grad = dict(dtype=1, act=0, dh=FAKE, ld_dh=16, x=FAKE, rows=4, n_in=8, ld_x=8, wg=FAKE, ld_g=8, wu=FAKE, ld_u=8, n_out=16,
                dx=FAKE, ld_dx=8, dg=FAKE, ld_dg=8, du=FAKE, ld_du=8, ws=FAKE, bytes=1 << 30)

    def call_grad(**kw):
        return nd._ffn_grad(*{**grad, **kw}.values(), None)

    for kw in (dict(dg=None), dict(du=None), dict(ld_dg=7), dict(ld_du=7), dict(ld_dx=7), dict(ld_dh=15), dict(dh=None), dict(x=None),
               dict(ws=None)):
        assert call_grad(**kw) == nd.E_ARG, kw
    assert call_grad(bytes=100) == nd.E_NOMEM
    assert call_grad(dx=None, dg=None, du=None) == nd.OK


def test_workspace_sizes_do_not_overflow():
    n = nd._sz()
    assert nd._norm_ws(0, 8, ctypes.byref(n)) == nd.OK
    assert nd._norm_ws(1 << 40, 1 << 40, ctypes.byref(n)) == nd.E_ARG
    assert nd._norm_ws(4, 8, None) == nd.E_ARG
    assert nd._ffn_ws(0, 1 << 22, 1 << 21, 1 << 21, 1, ctypes.byref(n)) == nd.OK and n.value > 1 << 45
    # a longer sequence of one head is cut into segments: their states need room
    assert nd._attn_ws(shape(n_seq=1, n_tokens=64, heads=1, kv_heads=1), 0, 0, ctypes.byref(n)) == nd.OK and n.value == 0
    assert nd._attn_ws(shape(n_seq=1, n_tokens=1 << 16, heads=1, kv_heads=1), 0, 0, ctypes.byref(n)) == nd.OK and n.value > 0


def test_launches_of_too_many_threads_are_refused():
    # an axis of a launch has fewer than 2^32 threads
    n = nd._sz()
    for s, packed in ((shape(n_seq=1 << 24, n_tokens=1 << 24, heads=1, kv_heads=1), 0),
                      (shape(n_seq=1 << 18, n_tokens=1 << 18, heads=64, kv_heads=64, dk=4, dv=4), 1)):
        for grad in (0, 1):
            assert nd._attn_ws(s, packed, grad, ctypes.byref(n)) == nd.E_UNSUPPORTED
    assert nd._attn_ws(shape(n_seq=(1 << 24) - 1, n_tokens=0, heads=1, kv_heads=1), 0, 1, ctypes.byref(n)) == nd.OK
    # many tokens are no reason: pieces grow with them
    assert nd._attn_ws(shape(n_seq=1, n_tokens=1 << 30, heads=16, kv_heads=16), 1, 1, ctypes.byref(n)) == nd.OK
    big = shape(n_seq=1 << 24, n_tokens=0, heads=1, kv_heads=1)
    assert nd._attn_step(big, heads(), heads(), heads(), FAKE, FAKE, 1 << 25, FAKE, heads(), None) == nd.E_UNSUPPORTED
    assert nd._norm_ws(8, 1 << 28, ctypes.byref(n)) == nd.E_UNSUPPORTED
    assert nd._norm_grad(0, FAKE, 1 << 28, FAKE, 1 << 28, 4, 1 << 28, None, FAKE, FAKE, FAKE, 1 << 28, FAKE, FAKE, FAKE,
                         1 << 50, None) == nd.E_UNSUPPORTED


# ---------------------------------------------------------------- the references
def differences(f, x, eps=1e-6):
    g = np.zeros_like(x)
    for i in np.ndindex(*x.shape):
        up, down = x.copy(), x.copy()
        up[i] += eps
        down[i] -= eps
        g[i] = (f(up) - f(down)) / (2 * eps)
    return g


def test_reference_gradients():
    rng = np.random.default_rng(0)
    r = lambda *s: rng.normal(size=s)
    x, w, b, dy = r(3, 5), r(5), r(5), r(3, 5)
    _, m, s = ref.norm(x, w, b, 1e-3)
    dx, dw, db = ref.norm_grad(dy, x, w, m, s)
    np.testing.assert_allclose(dx, differences(lambda t: (ref.norm(t, w, b, 1e-3)[0] * dy).sum(), x), atol=1e-7)
    np.testing.assert_allclose(dw, differences(lambda t: (ref.norm(x, t, b, 1e-3)[0] * dy).sum(), w), atol=1e-7)
    np.testing.assert_allclose(db, differences(lambda t: (ref.norm(x, w, t, 1e-3)[0] * dy).sum(), b), atol=1e-7)
    q, k, v, s0, do, ds = r(7, 4, 2), r(7, 2, 2), r(7, 2, 3), r(3, 4, 2, 3), r(7, 4, 3), r(3, 4, 2, 3)
    g, bounds = np.array([-0.3, 0.0, -1.0, -0.01]), [0, 3, 3, 7]

    def loss(q, k, v, s0):
        o, last = ref.attention(q, k, v, g, 0.4, bounds, s0)
        return (o * do).sum() + (last * ds).sum()

    got = ref.attention_grad(do, q, k, v, g, 0.4, bounds, s0, ds)
    args = [q, k, v, s0]
    for i in range(4):
        np.testing.assert_allclose(got[i], differences(lambda t: loss(*args[:i], t, *args[i + 1:]), args[i]), atol=1e-7)
    x, wg, wu, dh = r(3, 4), r(5, 4), r(5, 4), r(3, 5)
    for name in ("silu", "gelu", "sigmoid", "relu"):
        got = ref.ffn_grad(dh, x, wg, wu, name)
        args = [x, wg, wu]
        for i in range(3):
            want = differences(lambda t: (ref.ffn(*args[:i], t, *args[i + 1:], name) * dh).sum(), args[i])
            np.testing.assert_allclose(got[i], want, atol=1e-6)


def test_reference_attention_is_the_double_sum():
    rng = np.random.default_rng(1)
    q, k, v = rng.normal(size=(6, 1, 3)), rng.normal(size=(6, 1, 3)), rng.normal(size=(6, 1, 2))
    o, last = ref.attention(q, k, v, np.array([-0.2]), 2.0, [0, 6])
    for i in range(6):
        want = sum(np.exp(-0.2 * (i - j)) * (q[i, 0] @ k[j, 0]) * v[j, 0] for j in range(i + 1))
        np.testing.assert_allclose(o[i, 0], 2.0 * want, rtol=1e-12)

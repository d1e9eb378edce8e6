"""The operators around the attention of an encoder block, without a GPU: what the C entry points refuse before anything
is enqueued, workspace sizes, and the references that the GPU tests compare with, pinned to differences."""
import ctypes

import numpy as np
import pytest

import rms_ref
from test_encoder_host import FAKE, differences

nd = pytest.importorskip("paper_2607_03574_amd")


def test_rms_refusals():
    ok = dict(dtype=0, x=FAKE, rows=4, n=8, ld_x=8, r=FAKE, ld_r=8, w=None, eps=1e-5, y=FAKE, ld_y=8, h=FAKE, ld_h=8, rstd=None)

    def call(**kw):
        return nd._rms(*{**ok, **kw}.values(), None)

    for kw in (dict(dtype=3), dict(dtype=-1), dict(rows=-1), dict(n=0), dict(ld_x=7), dict(ld_y=7), dict(ld_r=7), dict(ld_h=7),
               dict(eps=-1.0), dict(eps=float("nan")), dict(x=None), dict(y=None), dict(h=None), dict(rows=1 << 62, ld_x=1 << 62)):
        assert call(**kw) == nd.E_ARG, kw
        assert "ndvm_rms_norm" in nd.last_error()
    assert call(rows=0, x=None, y=None, h=None) == nd.OK
    eight = dict(dtype=0, x=FAKE, rows=4, n=8, ld_x=8, r=FAKE, ld_r=8, w=None, eps=1e-5, y=FAKE, ld_y=8, scale=FAKE, h=FAKE, ld_h=8)
    for kw in (dict(scale=None), dict(y=None), dict(h=None), dict(ld_y=7), dict(eps=float("inf"))):
        assert nd._rms_8bit(*{**eight, **kw}.values(), None) == nd.E_ARG, kw
    rows = dict(dtype=0, x=FAKE, rows=4, n=8, ld_x=8, y=FAKE, ld_y=8, scale=FAKE)
    for kw in (dict(scale=None), dict(x=None), dict(ld_x=7), dict(dtype=4), dict(n=-1)):
        assert nd._quantize(*{**rows, **kw}.values(), None) == nd.E_ARG, kw
    assert nd._quantize(*{**rows, "rows": 0, "scale": None}.values(), None) == nd.OK


def test_rms_grad_refusals():
    ok = dict(dtype=1, dy=FAKE, ld_dy=8, h=FAKE, ld_h=8, rows=4, n=8, w=None, rstd=FAKE, dh=FAKE, ld_dh=8, dx=FAKE, ld_dx=8,
              dw=FAKE, ws=FAKE, bytes=1 << 20)

    def call(**kw):
        return nd._rms_grad(*{**ok, **kw}.values(), None)

    for kw in (dict(dtype=5), dict(rstd=None), dict(dy=None), dict(h=None), dict(ld_dx=7), dict(ld_dh=7), dict(ws=None),
               dict(ws=FAKE + 2)):
        assert call(**kw) == nd.E_ARG, kw
    assert call(bytes=16) == nd.E_NOMEM
    assert call(dx=None, dw=None, ws=None, bytes=0) == nd.OK       # nothing wanted
    assert call(n=1 << 28, ld_dy=1 << 28, ld_h=1 << 28, ld_dh=1 << 28, ld_dx=1 << 28, bytes=1 << 50) == nd.E_UNSUPPORTED
    n = nd._sz()
    assert nd._rms_ws(0, 8, ctypes.byref(n)) == nd.OK
    assert nd._rms_ws(1 << 40, 1 << 40, ctypes.byref(n)) == nd.E_ARG
    assert nd._rms_ws(8, 1 << 28, ctypes.byref(n)) == nd.E_UNSUPPORTED
    assert nd._rms_ws(4, 8, None) == nd.E_ARG


def test_reference_rms_gradient():
    rng = np.random.default_rng(0)
    h, w, dy, dh = (rng.normal(size=s) for s in ((3, 5), (5,), (3, 5), (3, 5)))
    _, rstd = rms_ref.rms(h, w, 1e-3)
    dx, dw = rms_ref.rms_grad(dy, h, w, rstd, dh)
    np.testing.assert_allclose(dx, differences(lambda t: (rms_ref.rms(t, w, 1e-3)[0] * dy).sum() + (t * dh).sum(), h), atol=1e-7)
    np.testing.assert_allclose(dw, differences(lambda t: (rms_ref.rms(h, t, 1e-3)[0] * dy).sum(), w), atol=1e-7)

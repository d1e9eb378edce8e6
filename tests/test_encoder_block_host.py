"""The operators around the attention of an encoder block, without a GPU: what the C entry points refuse before anything
is enqueued, workspace sizes, and the references that the GPU tests compare with, pinned to differences."""
import ctypes
import importlib.util
import os
import subprocess

import numpy as np
import pytest

import linear_ref
import rms_ref
from conftest import ROOT
from linear_sizes import LINEAR_CUTS
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


def test_linear_refusals():
    # (few rows need no workspace)
    ok = dict(dtype=1, act=4, x=FAKE, rows=400, n_in=8, ld_x=8, w=FAKE, ld_w=8, n_out=16, b=None, r=FAKE, ld_r=16, y=FAKE, ld_y=16,
              ws=FAKE, bytes=1 << 30)

    def call(**kw):
        return nd._linear(*{**ok, **kw}.values(), None)

    for kw in (dict(dtype=7), dict(act=5), dict(act=-1), dict(rows=-1), dict(n_in=0), dict(n_out=0), dict(ld_x=7), dict(ld_w=7),
               dict(ld_r=15), dict(ld_y=15), dict(x=None), dict(w=None), dict(y=None), dict(ws=None)):
        assert call(**kw) == nd.E_ARG, kw
    for kw in (dict(rows=1 << 23), dict(n_in=1 << 22, ld_x=1 << 22, ld_w=1 << 22), dict(n_out=1 << 22, ld_y=1 << 22, ld_r=1 << 22)):
        assert call(**kw) == nd.E_UNSUPPORTED, kw
    assert call(bytes=10) == nd.E_NOMEM
    assert call(rows=0, x=None, y=None) == nd.OK
    grad = dict(dtype=1, act=0, dy=FAKE, ld_dy=16, x=FAKE, rows=4, n_in=8, ld_x=8, w=FAKE, ld_w=8, n_out=16, b=None, dx=FAKE, ld_dx=8,
                dw=FAKE, ld_dw=8, db=FAKE, ws=FAKE, bytes=1 << 30)

    def call_grad(**kw):
        return nd._linear_grad(*{**grad, **kw}.values(), None)

    for kw in (dict(ld_dw=7), dict(ld_dx=7), dict(ld_dy=15), dict(dy=None), dict(x=None), dict(w=None), dict(ws=None), dict(act=9)):
        assert call_grad(**kw) == nd.E_ARG, kw
    assert call_grad(bytes=100) == nd.E_NOMEM
    assert call_grad(dx=None, dw=None, db=None) == nd.OK
    eight = dict(dtype=1, act=4, x=FAKE, sx=FAKE, rows=400, n_in=8, ld_x=8, w=FAKE, sw=FAKE, ld_w=8, n_out=16, b=None, r=None, ld_r=0,
                 y=FAKE, ld_y=16, ws=FAKE, bytes=1 << 30)

    def call_8bit(**kw):
        return nd._linear8(*{**eight, **kw}.values(), None)

    for kw in (dict(sx=None), dict(sw=None), dict(ld_x=7), dict(r=FAKE, ld_r=15), dict(y=None), dict(ws=None), dict(dtype=3)):
        assert call_8bit(**kw) == nd.E_ARG, kw
    assert call_8bit(bytes=10) == nd.E_NOMEM and call_8bit(dtype=0) == nd.E_UNSUPPORTED
    assert call_8bit(rows=0, x=None, sx=None, sw=None, y=None) == nd.OK
    n = nd._sz()
    assert nd._linear_ws(0, 0, 1 << 22, 1 << 21, 1 << 21, 1, ctypes.byref(n)) == nd.OK and n.value > 1 << 44
    assert nd._linear_ws(0, 0, 64, 1 << 21, 1 << 21, 0, ctypes.byref(n)) == nd.OK and n.value == 0
    assert nd._linear8_ws(1 << 22, 1 << 21, 1 << 21, ctypes.byref(n)) == nd.OK and n.value > 1 << 43
    assert nd._linear8_ws(1, 0, 1, ctypes.byref(n)) == nd.E_ARG and nd._linear_ws(0, 5, 1, 1, 1, 0, ctypes.byref(n)) == nd.E_ARG


def test_reference_linear_gradient():
    torch = pytest.importorskip("torch")
    rng = np.random.default_rng(2)
    x, w, b, dy = (rng.normal(size=s) for s in ((3, 4), (5, 4), (5,), (3, 5)))
    t = torch.tensor
    for name in linear_ref.ACTS:
        got = linear_ref.linear_grad(t(dy), t(x), t(w), t(b), name)
        args = [x, w, b]
        for i in range(3):
            want = differences(lambda v: float((linear_ref.linear(*(t(a) for a in args[:i] + [v] + args[i + 1:]), name) * t(dy)).sum()), args[i])
            np.testing.assert_allclose(got[i].numpy(), want, atol=1e-6)


CUTS = '''
#include "%s"
extern "C" void cuts(int dtype, int64_t rows, int64_t n_in, int64_t n_out, int64_t *to) {
    const auto g = ndvm::ops::linear_cut(dtype, rows, n_in, n_out);
    const auto p = ndvm::ops::linear_pieces(dtype, rows, n_in, n_out);
    const int64_t all[] = {g.ba, g.bb, g.splits, p.tile, p.dx, p.dw};
    for (int i = 0; i < 6; ++i) to[i] = all[i];
}
'''


@pytest.fixture(scope="module")
def cuts(tmp_path_factory):
    spec = importlib.util.spec_from_file_location("_b", os.path.join(ROOT, "paper_2607_03574_amd", "build.py"))
    b = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(b)
    if not os.path.exists(b.HIPCC):
        pytest.skip("no compiler")
    d = tmp_path_factory.mktemp("cuts")
    (d / "cuts.cpp").write_text(CUTS % os.path.join(b.CSRC, "ffn_cut.h"))
    subprocess.run([b.HIPCC, "-O1", "-std=c++17", "-shared", "-fPIC", str(d / "cuts.cpp"), "-o", str(d / "cuts.so")],
                   check=True, capture_output=True)
    f = ctypes.CDLL(str(d / "cuts.so")).cuts
    f.argtypes, f.restype = [ctypes.c_int] + [ctypes.c_int64] * 3 + [ctypes.c_void_p], None

    def call(dtype, *size):
        to = (ctypes.c_int64 * 6)()
        f(dtype, *size, to)
        return tuple(to)

    return call


@pytest.mark.parametrize("dtype", [0, 1])
def test_linear_sizes_cover_every_cut(cuts, dtype):
    taken = [cuts(dtype, *size) for size in LINEAR_CUTS]
    assert {(a, b, s > 1) for a, b, s, *_ in taken} == {(256, 256, False), (256, 128, False), (128, 128, False), (128, 128, True)}
    assert {(t, x > 1, w > 1) for *_, t, x, w in taken} == {(t, x, w) for t in (128, 256) for x in (False, True) for w in (False, True)}
    # the 8-bit form takes the tiles of half as long a sum of 16 bits
    eight = [cuts(1, rows, (n_in + 1) // 2, n_out) for rows, n_in, n_out in LINEAR_CUTS]
    assert {(a, b, s > 1) for a, b, s, *_ in eight} == {(256, 256, False), (256, 128, False), (128, 128, False), (128, 128, True)}


def test_delta_refusals():
    def shape(**kw):
        return nd._DeltaShape(*{**dict(dtype=1, n_seq=2, n_tokens=8, heads=4, qk_heads=2, dk=8, dv=16, scale=1.0), **kw}.values())

    h, none = nd._Heads(FAKE, 0, 64, 16), nd._Heads(None, 0, 0, 0)
    far, apart = nd._Heads(FAKE, 0, -1, 16), nd._Heads(FAKE, 0, 1 << 24, 16)

    def forward(s=None, q=h, v=h, g=h, o=h, off=FAKE, ws=FAKE, size=1 << 30):
        return nd._delta(s or shape(), q, h, v, g, h, off, None, o, None, ws, size, None)

    def gradient(s=None, do=h, dq=h, dg=h, off=FAKE, ws=FAKE, size=1 << 30):
        return nd._delta_grad(s or shape(), h, h, h, h, h, off, None, do, None, dq, none, none, dg, none, None, ws, size, None)

    for call in (forward, gradient):
        for kw in (dict(dtype=3), dict(n_seq=-1), dict(heads=0), dict(qk_heads=3), dict(dk=0), dict(dv=0), dict(scale=float("nan")),
                   dict(n_tokens=-1), dict(n_seq=0)):
            assert call(shape(**kw)) == nd.E_ARG, kw
        for kw in (dict(dk=257), dict(dv=257), dict(heads=1 << 16, qk_heads=1), dict(n_tokens=(1 << 30) + 1), dict(n_seq=1 << 24)):
            assert call(shape(**kw)) == nd.E_UNSUPPORTED, kw
        assert call(shape(n_tokens=9), off=None) == nd.E_ARG
        assert call(size=100) == nd.E_NOMEM and call(ws=None) == nd.E_ARG
        assert call(shape(n_seq=0, n_tokens=0)) == nd.OK
        assert nd.last_error()
    for kw in (dict(q=none), dict(v=far), dict(g=none), dict(o=none), dict(o=far)):
        assert forward(**kw) == nd.E_ARG, kw
    assert forward(v=apart) == forward(o=apart) == gradient(do=apart) == nd.E_UNSUPPORTED
    assert gradient(do=none) == nd.E_ARG and gradient(dq=far) == nd.E_ARG and gradient(dq=none, dg=none) == nd.OK

    def step(s=None, q=h, o=h, state=FAKE, n=2, slots=None):
        return nd._delta_step(s or shape(), q, h, h, h, h, state, n, slots, o, None)

    assert step(q=none) == nd.E_ARG and step(o=far) == nd.E_ARG and step(state=None) == nd.E_ARG and step(n=1) == nd.E_ARG
    assert step(shape(n_seq=0)) == nd.OK and step(shape(dk=300)) == nd.E_UNSUPPORTED and step(n=-1, slots=FAKE) == nd.E_ARG
    n = nd._sz()
    assert nd._delta_ws(shape(), 1, 0, ctypes.byref(n)) == nd.OK
    less = n.value
    assert nd._delta_ws(shape(), 1, 1, ctypes.byref(n)) == nd.OK and n.value > less
    assert nd._delta_ws(shape(heads=65535, qk_heads=65535, n_seq=1, n_tokens=1 << 12, dk=256, dv=256), 0, 1, ctypes.byref(n)) == nd.OK
    assert n.value > 1 << 40
    assert nd._delta_ws(shape(heads=65535, qk_heads=65535, n_seq=1, n_tokens=1 << 13), 0, 1, ctypes.byref(n)) == nd.E_UNSUPPORTED
    many = shape(n_seq=1 << 23, n_tokens=0, heads=1, qk_heads=1)
    assert nd._delta_ws(many, 1, 0, ctypes.byref(n)) == nd.OK and nd._delta_ws(many, 1, 1, ctypes.byref(n)) == nd.E_UNSUPPORTED
    assert gradient(many) == nd.E_UNSUPPORTED
    assert nd._delta_ws(shape(), 1, 1, None) == nd.E_ARG


def test_reference_delta_gradient():
    import delta_ref
    rng = np.random.default_rng(3)
    bounds, shapes = [0, 4, 4, 6], ((6, 1, 3), (6, 1, 3), (6, 2, 2), (6, 2), (6, 2), (3, 2, 3, 2))
    args = [rng.normal(size=s) for s in shapes]
    args[3], args[4] = -np.abs(args[3]), np.abs(args[4])
    do, ds = rng.normal(size=(6, 2, 2)), rng.normal(size=shapes[5])

    def loss(*x):
        o, last, _, _ = delta_ref.attention(*x[:5], 0.7, bounds, x[5])
        return (o * do).sum() + (last * ds).sum()

    got = delta_ref.attention_grad(do, *args[:5], 0.7, bounds, args[5], ds)
    for i in range(6):
        want = differences(lambda v: loss(*args[:i], v, *args[i + 1:]), args[i])
        np.testing.assert_allclose(got[i], want, atol=1e-6)

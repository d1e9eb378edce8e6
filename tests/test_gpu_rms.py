"""Root-mean-square norm with a residual, its gradient and its 8-bit result, and rows in 8 bits, against references in
64 bits within derived bounds, at the sizes, layouts and values where they can go wrong."""
import numpy as np
import pytest

import rms_ref as ref
from encoder_ref import F32, UNIT
from test_gpu_encoder import KINDS, TYPE, check, make, values

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

SIZES = [(1, 1), (3, 17), (5, 130), (300, 257), (33, 1000), (7, 2048), (600, 64), (9, 4100), (4, 8192), (3, 20001)]
EPS = 1e-3


@pytest.fixture(scope="module")
def nd():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2607_03574_amd as m
    return m


def case(rows, n, kind, seed):
    normal = make(rows * seed + n)
    return (normal(rows, n, kind=kind, scale=1.5, shift=0.5), normal(rows, n, kind=kind),
            normal(n, kind=kind, scale=0.3, shift=1.0), normal(rows, n, kind=kind))


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("rows,n", SIZES)
def test_rms_norm(nd, kind, rows, n):
    (x, xv), (r, rv), (w, wv), _ = case(rows, n, kind, 31)
    for we, re in ((w, r), (None, r), (w, None), (None, None)):
        y, h, rstd = nd.rms_norm(x, we, re, EPS)
        if re is None:
            assert h is x
        else:       # the sum as torch rounds it
            assert torch.equal(h, (x.float() + r.float()).to(TYPE[kind]))
        wy, wr = ref.rms(values(h), None if we is None else wv, EPS)
        check(rstd, wr, (n + 16) * F32 * wr)
        check(y, wy, ref.rms_bound(wy, n, kind), (we is None, re is None))


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("rows,n", SIZES)
def test_rms_norm_grad(nd, kind, rows, n):
    (h, hv), (dh, dhv), (w, wv), (dy, dyv) = case(rows, n, kind, 37)
    rstd = torch.tensor(ref.rms(hv, None, EPS)[1]).float().cuda()
    for we, de in ((w, dh), (None, dh), (w, None)):
        wt, dt = None if we is None else wv, None if de is None else dhv
        dx, dw = nd.rms_norm_grad(dy, h, we, rstd, de)
        wx, ww = ref.rms_grad(dyv, hv, wt, values(rstd), dt)
        bx, bw = ref.rms_grad_bounds(dyv, hv, wt, values(rstd), dt, kind)
        check(dx, wx, bx, "dx")
        check(dw, ww, bw, "dw")
        # what is not wanted is not needed for the rest; the same bits in every run
        only = nd.rms_norm_grad(dy, h, we, rstd, de, need_weight=False)
        assert only[1] is None and torch.equal(only[0], dx)
        again = nd.rms_norm_grad(dy, h, we, rstd, de, need_input=False)
        assert again[0] is None and torch.equal(again[1], dw)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("rows,n", SIZES)
def test_rows_in_8_bits(nd, kind, rows, n):
    (x, xv), (r, rv), (w, wv), _ = case(rows, n, kind, 41)
    y, scale = nd.quantize_rows(x)
    assert y.dtype == torch.float8_e4m3fn and y.shape == x.shape
    want = ref.row_scale(xv)
    check(scale, want, F32 * want)
    check(y.double() * scale.double()[:, None], xv, ref.rows_8bit_bound(xv, want, 0.0))
    # to nearest, as torch rounds the scaled values, wherever they are clear of the middle between two
    scaled = x.double() / scale.double()[:, None]
    a, b = (scaled * (1 + d * 4 * F32) for d in (-1, 1))
    clear = a.float().to(torch.float8_e4m3fn).float() == b.float().to(torch.float8_e4m3fn).float()
    assert torch.equal(y.float()[clear], a.float().to(torch.float8_e4m3fn).float()[clear])
    assert float(y.float().abs().max()) == 448.0
    for we, re in ((w, r), (None, None)):
        y, scale, h = nd.rms_norm_8bit(x, we, re, EPS)
        plain, h2, _ = nd.rms_norm(x, we, re, EPS)
        assert torch.equal(h, h2)
        wy, _ = ref.rms(values(h), None if we is None else wv, EPS)
        e = (n + 16) * F32 * np.abs(wy)
        ws = ref.row_scale(wy)
        check(scale, ws, (n + 20) * F32 * ws)
        check(y.double() * scale.double()[:, None], wy, ref.rows_8bit_bound(wy, ws, e))


def test_8_bit_rows_that_are_zero_tiny_large_or_not_finite(nd):
    x = torch.zeros(7, 70, device="cuda")
    x[1] = 1e-40
    x[2, 3] = 3e38
    x[2, 4] = -1e36
    x[3, 5] = float("nan")
    x[3, 6] = 1.0
    x[4, 1] = 1e-38
    x[5] = torch.linspace(-448, 448, 70)
    y, scale = nd.quantize_rows(x)
    tiny = 2.0 ** -126
    assert scale[0] == tiny and torch.all(y[0].float() == 0)
    assert scale[1] == tiny and torch.all(y[1].float() == 2.0 ** -7)       # 1e-40 / 2^-126 = 4.36 steps of 2^-9
    assert y[2, 3].float() == 448.0 and y[2, 4].float() < 0 and scale[2] > 6e35
    assert torch.isnan(scale[3])
    assert scale[4] == tiny and y[4, 1].float() == 0.875       # 1e-38 / 2^-126 = 0.8507 = 13.6 steps of 2^-4
    assert scale[5] == 1.0 and torch.equal(y[5].float(), x[5].to(torch.float8_e4m3fn).float())
    assert scale[6] == tiny


def test_rows_with_strides_and_many_rows(nd):
    normal = make(5)
    big, bv = normal(2100, 77, kind="bf16", shift=3.0)
    res, rv = normal(2100, 91, kind="bf16")
    x, r = big[:, 3:70], res[:, 11:78]           # rows start at odd places
    out = torch.full((2100, 80), -7.25, dtype=torch.bfloat16, device="cuda")
    y, h, rstd = nd.rms_norm(x, None, r, EPS, out=out[:, 5:72])
    wy, wr = ref.rms(values(h), None, EPS)
    check(y, wy, ref.rms_bound(wy, 67, "bf16"))
    assert torch.equal(h, (x.float() + r.float()).bfloat16()) and h.is_contiguous()
    assert torch.all(out[:, :5] == -7.25) and torch.all(out[:, 72:] == -7.25)
    dx, dw = nd.rms_norm_grad(out[:, 5:72], x, None, rstd, r)
    wx, ww = ref.rms_grad(values(y), bv[:, 3:70], None, values(rstd), rv[:, 11:78])
    bx, bw = ref.rms_grad_bounds(values(y), bv[:, 3:70], None, values(rstd), rv[:, 11:78], "bf16")
    check(dx, wx, bx)
    check(dw, ww, bw)
    y8, scale, _ = nd.rms_norm_8bit(x, None, r, EPS)
    one8, one, _ = nd.rms_norm_8bit(x[1234:1235], None, r[1234:1235], EPS)      # whatever the number of rows
    assert torch.equal(y8[1234:1235].float(), one8.float()) and torch.equal(scale[1234:1235], one)
    # a row with a NaN is NaN, and no other row
    x2 = x.clone()
    x2[3, 5] = float("nan")
    y2, s2, h2 = nd.rms_norm_8bit(x2, None, r, EPS)
    assert torch.isnan(s2[3]) and torch.isnan(y2[3].float()).all()
    keep = torch.arange(2100, device="cuda") != 3
    assert torch.equal(y2.float()[keep], y8.float()[keep]) and torch.equal(s2[keep], scale[keep])
    # leading axes, and a row that passes the caches by
    x3 = x.clone().view(21, 100, 67)
    y3, h3, r3 = nd.rms_norm(x3, None, r.clone().view(21, 100, 67), EPS)
    assert y3.shape == x3.shape and r3.shape == (21, 100) and torch.equal(y3.view(2100, 67), y)


@pytest.mark.parametrize("kind", ["bf16", "f32"])
def test_large_calls(nd, kind):
    # results that are marked as passing through: the same bits as a few rows alone
    rows, n = (40000, 1024) if kind == "bf16" else (20000, 1024)
    gen = torch.Generator(device="cuda").manual_seed(7)
    x, r, dy = (torch.randn(rows, n, generator=gen, device="cuda").to(TYPE[kind]) for _ in range(3))
    w = torch.randn(n, generator=gen, device="cuda").to(TYPE[kind])
    y, h, rstd = nd.rms_norm(x, w, r)
    y8, scale, h8 = nd.rms_norm_8bit(x, w, r)
    dx, dw = nd.rms_norm_grad(dy, h, w, rstd, r)
    part = slice(rows - 50, rows)
    z, hz, rz = nd.rms_norm(x[part], w, r[part])
    z8, sz, _ = nd.rms_norm_8bit(x[part], w, r[part])
    assert torch.equal(y[part], z) and torch.equal(h[part], hz) and torch.equal(rstd[part], rz) and torch.equal(h8, h)
    assert torch.equal(y8[part].float(), z8.float()) and torch.equal(scale[part], sz)
    assert torch.equal(dx[part], nd.rms_norm_grad(dy[part], h[part], w, rstd[part], r[part])[0])
    terms = dy.double() * h.double() * rstd.double()[:, None]
    bound = UNIT[kind] * terms.sum(0).abs() * 1.01 + (rows + 16) * F32 * terms.abs().sum(0)
    assert torch.all((dw.double() - terms.sum(0)).abs() <= bound)


def test_no_rows(nd):
    x = torch.empty(0, 40, device="cuda")
    y, h, rstd = nd.rms_norm(x, None, x)
    assert y.shape == (0, 40) and rstd.shape == (0,)
    dx, dw = nd.rms_norm_grad(x, x, None, rstd)
    assert dx.shape == (0, 40) and torch.all(dw == 0)
    y8, scale, _ = nd.rms_norm_8bit(x)
    assert y8.shape == (0, 40) and scale.shape == (0,)


def test_autograd(nd):
    from paper_2607_03574_amd import torch_api
    gen = torch.Generator(device="cuda").manual_seed(3)
    x, r = (torch.randn(6, 9, 33, generator=gen, device="cuda", requires_grad=True) for _ in range(2))
    w = torch.randn(33, generator=gen, device="cuda", requires_grad=True)
    a, b = (torch.randn(6, 9, 33, generator=gen, device="cuda") for _ in range(2))

    def plain(x, w, r):
        h = x.double() + r.double()
        return h * (h.square().mean(-1, keepdim=True) + 1e-5).rsqrt() * w.double(), h

    for use in ("both", "y", "h"):
        (y, h), (py, ph) = torch_api.rms_norm(x, w, r), plain(x, w, r)
        loss, pl = ({"both": (a * y).sum() + (b * h).sum(), "y": (a * y).sum(), "h": (b * h).sum()}[use] for y, h in ((y, h), (py, ph)))
        leaves = (x, r) if use == "h" else (x, r, w)
        for got, want in zip(torch.autograd.grad(loss, leaves), torch.autograd.grad(pl, leaves)):
            assert torch.allclose(got.double(), want.double(), rtol=0, atol=60 * 33 * F32 * float(want.abs().max() + 1))
    # the same tensor twice, strided, and nothing wanted of the weight
    t = torch.randn(33, 54, generator=gen, device="cuda").t().requires_grad_()
    y, h = torch_api.rms_norm(t, w.detach(), t)
    (g,) = torch.autograd.grad((y * a.view(54, 33)).sum() + h.sum(), t)
    py, ph = plain(t, w.detach(), t)
    (pg,) = torch.autograd.grad((py * a.view(54, 33)).sum() + ph.sum(), t)
    assert torch.allclose(g.double(), pg.double(), rtol=0, atol=60 * 33 * F32 * float(pg.abs().max() + 1))
    y = torch_api.rms_norm(x, w)
    assert torch.is_tensor(y) and y.requires_grad


def test_refusals(nd):
    x = torch.randn(4, 8, device="cuda")
    for kw in (dict(weight=torch.ones(7, device="cuda")), dict(residual=x[:3]), dict(residual=x[:, :7]), dict(out=x[:2])):
        with pytest.raises(ValueError):
            nd.rms_norm(x, **kw)
    for kw in (dict(weight=torch.ones(8)), dict(residual=x.bfloat16()), dict(residual=x.cpu())):
        with pytest.raises(TypeError):
            nd.rms_norm(x, **kw)
    with pytest.raises(TypeError):
        nd.quantize_rows(x.double())
    with pytest.raises(ValueError):
        nd.rms_norm_grad(x, x, None, torch.ones(4, device="cuda"), dh=x[:1])
    with pytest.raises(nd.NdvmError):
        nd.rms_norm(x, eps=-1.0)

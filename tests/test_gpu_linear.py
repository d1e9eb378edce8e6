"""Projections with bias, activation and residual, their gradient and their 8-bit form, against references in 64 bits
within derived bounds, at the sizes, layouts and values where they can go wrong."""
import pytest

import linear_ref as ref
from encoder_ref import F32
from linear_sizes import LINEAR_CUTS

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

TYPE = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
FEW = [(1, 1, 1), (3, 17, 5), (16, 130, 40), (17, 64, 33), (33, 200, 70), (64, 100, 513), (17, 4096, 1024), (2, 3001, 48)]


@pytest.fixture(scope="module")
def nd():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2607_03574_amd as m
    return m


def make(seed, kind):
    gen = torch.Generator(device="cuda").manual_seed(seed)

    def normal(*shape, scale=1.0):
        return (torch.randn(shape, generator=gen, device="cuda", dtype=torch.float64) * scale).to(TYPE[kind])

    return normal


def check(got, want, bound, what=""):
    error = (got.double() - want).abs()
    assert error.shape == bound.shape and bool((error <= bound).all()), (what, float((error / bound).nan_to_num(1e9).max()))


def near(got, want, rounded, what=""):
    """As near in norm as the roundings to the type are, or, in float, 1e-6: a part of an operand that was left out in
    some places shows here."""
    limit = 1e-6 * want.norm() if got.dtype == torch.float32 else 1.02 * (rounded - want).norm()
    assert (got.double() - want).norm() <= limit + 1e-30, (what, float((got.double() - want).norm() / want.norm()))


def dbl(t):
    return None if t is None else t.double()


@pytest.mark.parametrize("kind", list(TYPE))
@pytest.mark.parametrize("rows,n_in,n_out", FEW + LINEAR_CUTS)
def test_linear(nd, kind, rows, n_in, n_out):
    normal = make(rows + n_in, kind)
    x, w, b, r = normal(rows, n_in), normal(n_out, n_in, scale=n_in ** -0.5), normal(n_out, scale=0.5), normal(rows, n_out)
    acts = ref.ACTS if rows * n_in * n_out < 1 << 24 else ["silu"]
    for name, be, re in [(a, b, r) for a in acts] + [(None, None, None), ("gelu", None, r), (None, b, None)]:
        y = nd.linear(x, w, be, name, re)
        want = ref.linear(dbl(x), dbl(w), dbl(be), name, dbl(re))
        check(y, want, ref.linear_bound(dbl(x), dbl(w), dbl(be), name, dbl(re), kind), (name, be is None, re is None))
        if rows * n_out > 4000:
            near(y, want, want.to(y.dtype).double(), name)


@pytest.mark.parametrize("kind", list(TYPE))
@pytest.mark.parametrize("rows,n_in,n_out", FEW + LINEAR_CUTS)
def test_linear_grad(nd, kind, rows, n_in, n_out):
    normal = make(rows + n_in + 1, kind)
    x, w, b, dy = normal(rows, n_in), normal(n_out, n_in, scale=n_in ** -0.5), normal(n_out, scale=0.5), normal(rows, n_out)
    acts = ref.ACTS if rows * n_in * n_out < 1 << 24 else [None, "silu"]
    for name in acts:
        got = nd.linear_grad(dy, x, w, b, name)
        args = [t.double() for t in (dy, x, w, b)]
        want = ref.linear_grad(*args, name)
        for g, v, e, what in zip(got, want, ref.linear_grad_bounds(*args, name, kind), ("dx", "dw", "db")):
            check(g, v, e, (name, what))
        if name != "relu" and min(rows, n_in, n_out) > 10 and rows * n_in * n_out > 1 << 18:
            dz = (args[0] * ref.act(name, args[1] @ args[2].T + args[3])[1]).to(TYPE[kind]).double()
            for g, v, t, what in zip(got[:2], want, (dz @ args[2], dz.T @ args[1]), ("dx", "dw")):
                near(g, v, t.to(TYPE[kind]).double(), (name, what))
        # what is not wanted is not needed for the rest; the same bits in every run
        for i in range(3):
            only = nd.linear_grad(dy, x, w, b, name, *[j == i for j in range(3)])
            assert all((o is None) == (j != i) for j, o in enumerate(only)) and torch.equal(only[i], got[i])
    assert nd.linear_grad(dy, x, w, None, "silu")[2] is None


@pytest.mark.parametrize("kind", ["bf16", "f16"])
@pytest.mark.parametrize("rows,n_in,n_out", FEW + LINEAR_CUTS)
def test_linear_8bit(nd, kind, rows, n_in, n_out):
    """The matrix instructions for many rows cut, of eight products, what lies below 2^-13 of the largest one's power of
    two: 7 of them lose less than that, and the largest is part of the sum of magnitudes.  The slopes are at most 1.13."""
    cut = 1.13 * 7 * 2.0 ** -13 if rows > 64 else 0.0
    normal = make(rows + n_in + 2, kind)
    x, sx = nd.quantize_rows(normal(rows, n_in))
    w, sw = nd.quantize_rows(normal(n_out, n_in, scale=n_in ** -0.5))
    b, r = normal(n_out, scale=0.5), normal(rows, n_out)
    xd, wd = x.double() * sx.double()[:, None], w.double() * sw.double()[:, None]
    acts = ref.ACTS if rows * n_in * n_out < 1 << 24 else ["gelu"]
    for name, be, re in [(a, b, r) for a in acts] + [(None, None, None)]:
        y = nd.linear_8bit(x, sx, w, sw, be, name, re, dtype=TYPE[kind])
        want = ref.linear(xd, wd, dbl(be), name, dbl(re))
        check(y, want, ref.linear_bound(xd, wd, dbl(be), name, dbl(re), kind) + cut * (xd.abs() @ wd.abs().T), (name, be is None))
        if rows * n_out > 4000:
            near(y, want, want.to(y.dtype).double(), name)


@pytest.mark.parametrize("kind", list(TYPE))
@pytest.mark.parametrize("rows,n_in,n_out", [(5, 65, 40), (70, 65, 40), (300, 129, 257), (600, 64, 96)])
def test_whole_numbers_are_exact(nd, kind, rows, n_in, n_out):
    """Small whole numbers: every product and sum is exact, in 8 bits too, whatever the order and the layout of the
    operands in the instructions."""
    gen = torch.Generator(device="cuda").manual_seed(rows)
    whole = lambda *s: torch.randint(-3, 4, s, generator=gen, device="cuda").double()
    x, w, b, r = whole(rows, n_in), (whole(n_out, n_in) / 2).trunc(), whole(n_out), whole(rows, n_out)
    t = TYPE[kind]
    want = torch.relu(x @ w.T + b) + r
    assert torch.equal(nd.linear(x.to(t), w.to(t), b.to(t), "relu", r.to(t)).double(), want.to(t).double())
    dy = whole(rows, n_out)
    for g, v in zip(nd.linear_grad(dy.to(t), x.to(t), w.to(t), b.to(t), "relu"), ref.linear_grad(dy, x, w, b, "relu")):
        assert torch.equal(g.double(), v.to(t).double())
    if kind == "f32":
        return
    e4m3 = torch.float8_e4m3fn
    sx, sw = 2.0 ** torch.arange(rows, device="cuda").fmod(3).float(), 2.0 ** -torch.arange(n_out, device="cuda").fmod(4).float()
    y = nd.linear_8bit(x.float().to(e4m3), sx, w.float().to(e4m3), sw, b.to(t), "relu", r.to(t), dtype=t)
    want = torch.relu((x * sx.double()[:, None]) @ (w * sw.double()[:, None]).T + b) + r
    assert torch.equal(y.double(), want.to(t).double())


@pytest.mark.parametrize("kind", list(TYPE))
@pytest.mark.parametrize("rows", [7, 150])
def test_strides_and_alignment(nd, kind, rows):
    normal = make(3, kind)
    x, w, r, dy = normal(rows, 75)[:, 3:68], normal(51, 80)[:, 7:72], normal(rows, 90)[:, 1:52], normal(rows, 64)[:, 5:56]
    b = normal(60)[5:56]
    out = torch.full((rows, 60), -7.25, dtype=TYPE[kind], device="cuda")
    nd.linear(x, w, b, "silu", r, out=out[:, 3:54])
    args = [t.double() for t in (x, w, b)]
    check(out[:, 3:54], ref.linear(*args, "silu", r.double()), ref.linear_bound(*args, "silu", r.double(), kind))
    assert torch.all(out[:, :3] == -7.25) and torch.all(out[:, 54:] == -7.25)
    for name in ("gelu", None):
        for g, v, e in zip(nd.linear_grad(dy, x, w, b, name), ref.linear_grad(dy.double(), *args, name),
                           ref.linear_grad_bounds(dy.double(), *args, name, kind)):
            check(g, v, e, name)
    if kind == "f32":
        return
    x8, sx = nd.quantize_rows(x)
    w8, sw = nd.quantize_rows(w)
    wide = torch.zeros(rows, 91, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn)
    wide.view(torch.uint8)[:, 9:74] = x8.view(torch.uint8)
    y = nd.linear_8bit(wide[:, 9:74], sx, w8, sw, b, None, r, dtype=TYPE[kind])
    assert torch.equal(y, nd.linear_8bit(x8, sx, w8, sw, b, None, r, dtype=TYPE[kind]))


def test_values_that_are_not_finite_stay_in_their_rows_and_columns(nd):
    for rows in (9, 200):
        for kind in TYPE:
            normal = make(4, kind)
            x, w, b = normal(rows, 96), normal(40, 96), normal(40)
            y = nd.linear(x, w, b, "silu")
            x2, w2 = x.clone(), w.clone()
            x2[3, 95], w2[7, 0] = float("nan"), float("inf")
            z = nd.linear(x2, w2, b, "silu")
            assert torch.isnan(z[3]).all()
            keep = torch.ones_like(y, dtype=torch.bool)
            keep[3], keep[:, 7] = False, False
            assert torch.equal(y[keep], z[keep])


@pytest.mark.parametrize("scale", [2.0 ** -20, 1.0, 2.0 ** 12])
def test_gradient_range_of_half(nd, scale):
    """dz of halves that are tiny or large keeps its bits as an operand."""
    normal = make(6, "f16")
    x, w, b = normal(300, 64), normal(96, 64, scale=8.0), normal(96)
    dy = (normal(300, 96).double() * scale).to(torch.float16)
    args = [t.double() for t in (dy, x, w, b)]
    got, want = nd.linear_grad(dy, x, w, b, "sigmoid"), ref.linear_grad(*args, "sigmoid")
    for g, v, e, what in zip(got, want, ref.linear_grad_bounds(*args, "sigmoid", "f16"), ("dx", "dw", "db")):
        # results from 65520 on round to an infinity of half
        over = (v.abs() + e >= 65520) & torch.isinf(g) & (g.double().sign() == v.sign())
        assert not torch.isfinite(g)[v.abs() - e >= 65520].any()
        check(torch.where(over, v, g.double()), v, e, what)


def test_no_rows(nd):
    x, w, b = torch.empty(0, 40, device="cuda"), torch.ones(9, 40, device="cuda"), torch.ones(9, device="cuda")
    assert nd.linear(x, w, b, "gelu").shape == (0, 9)
    for kind in TYPE.values():
        for name in (None, "silu"):
            dx, dw, db = nd.linear_grad(torch.empty(0, 9, device="cuda", dtype=kind), x.to(kind), w.to(kind), b.to(kind), name)
            assert dx.shape == (0, 40) and torch.all(dw == 0) and torch.all(db == 0)
    x8, sx = nd.quantize_rows(x)
    w8, sw = nd.quantize_rows(w)
    assert nd.linear_8bit(x8, sx, w8, sw).shape == (0, 9)


def test_autograd(nd):
    from paper_2607_03574_amd import torch_api
    gen = torch.Generator(device="cuda").manual_seed(3)
    x, w, b, r = (torch.randn(*s, generator=gen, device="cuda", requires_grad=True) for s in ((6, 9, 33), (20, 33), (20,), (6, 9, 20)))
    dy = torch.randn(6, 9, 20, generator=gen, device="cuda")
    for name in ref.ACTS:
        y = torch_api.linear(x, w, b, name, r)
        plain = ref.linear(x.double(), w.double(), b.double(), name, r.double())
        got, want = (torch.autograd.grad((t * dy).sum(), (x, w, b, r)) for t in (y, plain))
        for g, v in zip(got, want):
            assert torch.allclose(g.double(), v.double(), rtol=0, atol=200 * F32 * float(v.abs().max() + 8))
    # transposed and expanded tensors, and only some gradients wanted
    wt = torch.randn(33, 20, generator=gen, device="cuda").t().requires_grad_()
    y = torch_api.linear(x.detach(), wt, None, "silu")
    (g,) = torch.autograd.grad(y.sum(), wt)
    (v,) = torch.autograd.grad(ref.linear(x.detach().double(), wt.double(), None, "silu").sum(), wt)
    assert torch.allclose(g.double(), v.double(), rtol=0, atol=200 * F32 * float(v.abs().max() + 8))
    (g,) = torch.autograd.grad(torch_api.linear(x.detach(), w.detach(), b).sum(), b)
    assert torch.all(g == 54)


def test_refusals(nd):
    x, w = torch.randn(4, 8, device="cuda"), torch.randn(6, 8, device="cuda")
    for kw in (dict(weight=w[:, :7]), dict(activation="tanh"), dict(bias=torch.ones(5, device="cuda")), dict(residual=x), dict(out=x),
               dict(weight=w[0])):
        with pytest.raises(ValueError):
            nd.linear(**{**dict(x=x, weight=w), **kw})
    for kw in (dict(weight=w.bfloat16()), dict(bias=torch.ones(6)), dict(residual=torch.ones(4, 6, device="cuda").half()), dict(x=x.double())):
        with pytest.raises(TypeError):
            nd.linear(**{**dict(x=x, weight=w), **kw})
    with pytest.raises(ValueError):
        nd.linear_grad(x, x, w)
    x8, sx = nd.quantize_rows(x)
    w8, sw = nd.quantize_rows(w)
    for a in ((x, sx, w8, sw), (x8, sx, w, sw), (x8, sx.double(), w8, sw)):
        with pytest.raises(TypeError):
            nd.linear_8bit(*a)
    for a in ((x8, sx[:3], w8, sw), (x8, sx, w8, sw[:2]), (x8, sx, w8[:, :4], sw)):
        with pytest.raises(ValueError):
            nd.linear_8bit(*a)
    with pytest.raises(TypeError):
        nd.linear_8bit(x8, sx, w8, sw, dtype=torch.float32)

"""The gated feed-forward in every way its products are cut (tiles, sums shared by several workgroups), and
relu's gradient, against plain references in 64 bits."""
import numpy as np
import pytest

import encoder_ref as ref
from encoder_sizes import FFN_CUTS

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

TYPE = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


@pytest.fixture(scope="module")
def nd():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2607_03574_amd as m
    return m


def values(t):
    return t.detach().double().cpu().numpy()


def to_type(a, kind):
    return values(torch.tensor(a).to(TYPE[kind]))


def check(got, want, rounded, bound, what):
    """Within the elementwise bound; and as near in norm as the roundings to the type are (done here on 64-bit values;
    float sums move few of them), or, in float, 1e-6: a part of an operand that was left out in some places shows in
    one or the other."""
    error = np.abs(values(got) - want)
    assert error.shape == bound.shape and np.all(error <= bound), (what, np.unravel_index(np.argmax(error - bound), error.shape))
    limit = 1e-6 * np.linalg.norm(want) if got.dtype == torch.float32 else 1.02 * np.linalg.norm(rounded - want)
    assert np.linalg.norm(error) <= limit, (what, np.linalg.norm(error), limit)


@pytest.mark.parametrize("kind", list(TYPE))
@pytest.mark.parametrize("rows,n_in,n_out", FFN_CUTS)
def test_every_cut(nd, kind, rows, n_in, n_out):
    rng = np.random.default_rng(rows + n_in + n_out)

    def normal(*shape, scale=1.0):
        t = torch.tensor(rng.normal(size=shape) * scale).to(TYPE[kind])
        return t.cuda(), values(t)

    (x, xv), (dh, dhv) = normal(rows, n_in), normal(rows, n_out)
    (wg, wgv), (wu, wuv) = (normal(n_out, n_in, scale=n_in ** -0.5) for _ in range(2))
    h = ref.ffn(xv, wgv, wuv, "silu")
    check(nd.gated_ffn(x, wg, wu), h, to_type(h, kind), ref.ffn_bound(xv, wgv, wuv, "silu", kind), "h")
    got = nd.gated_ffn_grad(dh, x, wg, wu)
    want = ref.ffn_grad(dhv, xv, wgv, wuv, "silu")
    # dg and du are rounded to the type, as operands, and the results
    g, u = xv @ wgv.T, xv @ wuv.T
    f, d = ref.act("silu", g)
    dg, du = to_type(dhv * u * d, kind), to_type(dhv * f, kind)
    rounded = [to_type(a, kind) for a in (dg @ wgv + du @ wuv, dg.T @ xv, du.T @ xv)]
    bounds = ref.ffn_grad_bound(dhv, xv, wgv, wuv, "silu", kind)
    for a, b, r, c, what in zip(got, want, rounded, bounds, ("dx", "dw_gate", "dw_up")):
        check(a, b, r, c, what)


@pytest.mark.parametrize("kind", list(TYPE))
@pytest.mark.parametrize("rows,n_in,n_out", [(3, 8, 5), (300, 64, 96), (700, 33, 1000)])
def test_relu_gradient(nd, kind, rows, n_in, n_out):
    """On small whole numbers every product and sum is exact, and g is 0 in many places: there no gradient goes through
    the gate, and the results are the exact ones rounded once."""
    rng = np.random.default_rng(n_out)
    xv, dhv = rng.integers(-2, 3, (rows, n_in)).astype(float), rng.integers(-1, 2, (rows, n_out)).astype(float)
    wgv, wuv = (rng.integers(-1, 2, (n_out, n_in)).astype(float) for _ in range(2))
    g, u = xv @ wgv.T, xv @ wuv.T
    assert (g == 0).mean() > 0.02 and np.abs(g).max() < 256 and np.abs(u).max() < 256      # dg and du have 8 bits
    x, dh, wg, wu = (torch.tensor(t).to(TYPE[kind]).cuda() for t in (xv, dhv, wgv, wuv))
    for a, b in zip(nd.gated_ffn_grad(dh, x, wg, wu, "relu"), ref.ffn_grad(dhv, xv, wgv, wuv, "relu")):
        assert np.array_equal(values(a), values(torch.tensor(b).to(TYPE[kind])))
    # a gate that is 0 everywhere: nothing through it, and the other weight's gradient is 0 with it
    for a in nd.gated_ffn_grad(dh, x, torch.zeros_like(wg), wu, "relu"):
        assert torch.all(a == 0)

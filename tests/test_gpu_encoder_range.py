"""The gradient of the gated feed-forward in half where dg = dh u act'(g) and du = dh act(g) leave half's
range on the way, large or small, and the results do not.

Limits: dg and du are rounded to 11 bits as operands (times the power of two that brings the largest
value that is finite into range), the result once more.  Both roundings are done here on the 64-bit values; what else a
kernel loses, in float sums, moves one rounding in some hundreds by one place: 2% in norm.  A
result past 65504 is an infinity, in half as in the 64-bit value rounded to it.
"""
import numpy as np
import pytest

import encoder_ref as ref

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

# sizes whose sums are shared by several workgroups, and not; one tile and several
SIZES = [(70, 2100, 200), (300, 64, 200), (33, 40, 8), (700, 136, 1500)]


@pytest.fixture(scope="module")
def nd():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2607_03574_amd as m
    return m


def values(t):
    return t.detach().double().cpu().numpy()


def half(rng, *shape, scale=1.0):
    t = torch.tensor(rng.normal(size=shape) * scale).half()
    assert torch.isfinite(t).all()
    return t.cuda(), values(t)


def to_half(a):
    return values(torch.tensor(a).half())


def gradients(dh, x, wg, wu, name):
    """In 64 bits, and with the two roundings."""
    g, u = x @ wg.T, x @ wu.T
    f, d = ref.act(name, g)
    dg, du = dh * u * d, dh * f
    top = max((np.abs(t[np.isfinite(t)]).max(initial=0.0) for t in (dg, du)))
    e = np.floor(np.log2(top)) if top else 0.0
    scale = 1.0 if 0 <= e < 15 else 2.0 ** (14 - e)
    rg, ru = to_half(dg * scale) / scale, to_half(du * scale) / scale
    return ((dg @ wg + du @ wu, to_half(rg @ wg + ru @ wu)), (dg.T @ x, to_half(rg.T @ x)), (du.T @ x, to_half(ru.T @ x)))


def in_range(want):
    return np.abs(want) < 65504 * (1 - 2.0 ** -9)       # but for what rounds to the end of the range


def close(got, both, what):
    """As near as the roundings where half holds the result, an infinity where it does not."""
    got, (want, rounded) = values(got), both
    held, past = in_range(want), np.abs(want) > 65520 * (1 + 2.0 ** -9)
    assert np.array_equal(got[past], np.sign(want[past]) * np.inf), what
    error, limit = (np.linalg.norm(t[held] - want[held]) for t in (got, rounded))
    assert error <= 1.02 * limit, (what, error, limit)


@pytest.mark.parametrize("rows,n_in,n_out", SIZES)
# standard deviations of dh, x and the weights (times n_in^-0.5): dg and du past 65504 with dx in range, with the
# weights' gradients in range; both far below 2^-24 on the way
@pytest.mark.parametrize("of_dh,of_x,of_w", [(3000.0, 3000.0, 0.03), (3000.0, 0.002, 30000.0), (2.0 ** -17, 0.5, 0.25), (2.0 ** -12, 2.0 ** -4, 2.0 ** -3)])
def test_gated_ffn_grad(nd, rows, n_in, n_out, of_dh, of_x, of_w):
    rng = np.random.default_rng(rows)
    dh, dhv = half(rng, rows, n_out, scale=of_dh)
    x, xv = half(rng, rows, n_in, scale=of_x)
    wg, wgv = half(rng, n_out, n_in, scale=of_w * n_in ** -0.5)
    wu, wuv = half(rng, n_out, n_in, scale=of_w * n_in ** -0.5)
    got = nd.gated_ffn_grad(dh, x, wg, wu, "sigmoid")
    compared = 0
    for a, b, what in zip(got, gradients(dhv, xv, wgv, wuv, "sigmoid"), ("dx", "dw_gate", "dw_up")):
        if in_range(b[0]).mean() > 0.99:        # else the rest are differences of sums that are out of range
            close(a, b, what)
            compared += 1
    assert compared


@pytest.mark.parametrize("rows,n_in,n_out", SIZES)
def test_values_that_are_not_finite_do_not_scale_the_others(nd, rows, n_in, n_out):
    rng = np.random.default_rng(1)
    dh, dhv = half(rng, rows, n_out, scale=2.0 ** -17)
    x, xv = half(rng, rows, n_in)
    (wg, wgv), (wu, wuv) = (half(rng, n_out, n_in, scale=n_in ** -0.5) for _ in range(2))
    want, rounded = gradients(dhv, xv, wgv, wuv, "silu")[0]
    for bad in (float("inf"), float("nan")):
        dh2 = dh.clone()
        dh2[5, 3] = bad
        dx = nd.gated_ffn_grad(dh2, x, wg, wu, need_weight=False)[0]
        keep = np.arange(rows) != 5
        assert not torch.isfinite(dx[5]).any()
        close(dx[torch.tensor(keep)], (want[keep], rounded[keep]), "dx")


def test_replays_find_the_range_anew(nd):
    """A captured call on new values: what one replay found does not stay for the next."""
    rng = np.random.default_rng(2)
    rows, n_in, n_out = 150, 64, 96
    x, wg, wu = (half(rng, *s, scale=c)[0] for s, c in (((rows, n_in), 40.0), ((n_out, n_in), 0.02), ((n_out, n_in), 0.02)))
    dh = torch.zeros(rows, n_out, dtype=torch.float16, device="cuda")
    nd.gated_ffn_grad(dh, x, wg, wu)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = nd.gated_ffn_grad(dh, x, wg, wu)
    for scale in (2.0 ** 15, 2.0 ** -15, 1.0, 0.0, 2.0 ** -15):
        dh.copy_(torch.tensor(rng.uniform(-1, 1, (rows, n_out)) * scale))
        graph.replay()
        torch.cuda.synchronize()
        want = nd.gated_ffn_grad(dh, x, wg, wu)
        assert all(torch.equal(a, b) for a, b in zip(got, want))
        exact = gradients(*(values(t) for t in (dh, x, wg, wu)), "silu")
        for a, b, what in zip(got, exact, ("dx", "dw_gate", "dw_up")):
            if in_range(b[0]).mean() > 0.99:
                close(a, b, what)

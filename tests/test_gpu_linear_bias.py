"""The bias's gradient of a projection is a sum in float of dz as it is formed, not of dz as it is rounded for the products:
against 64 bits, elementwise within a bound without that rounding, and as near in norm as the result's own rounding."""
import pytest

import linear_ref as ref
from encoder_ref import F32, TINY, UNIT
from linear_sizes import LINEAR_CUTS
from test_gpu_linear import FEW, TYPE, check, make, near

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def nd():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2607_03574_amd as m
    return m


def bias_bound(dy, x, w, b, name, kind):
    """linear_grad_bounds without the rounding of dz: what its float value may be off by, what a sum over the rows in float
    may lose, and the result's rounding."""
    z = x @ w.T + b
    slope = ref.act(name, z)[1]
    dz, e = (dy * slope).abs(), torch.zeros_like(z)
    if name is not None:
        ez = ref.z_error(x, w, b)
        e = dy.abs() * (0.8 * ez + 16 * F32 * (1 + z.abs()) if name != "relu" else (z.abs() <= ez).double())
    e = e.sum(0) + (x.shape[0] + 80) * F32 * (dz + e).sum(0)
    return UNIT[kind] * ((dy * slope).sum(0).abs() + e) + e + TINY[kind]


@pytest.mark.parametrize("kind", list(TYPE))
@pytest.mark.parametrize("rows,n_in,n_out", FEW + LINEAR_CUTS)
def test_bias_gradient(nd, kind, rows, n_in, n_out):
    normal = make(rows + n_in + 5, kind)
    x, w, b, dy = normal(rows, n_in), normal(n_out, n_in, scale=n_in ** -0.5), normal(n_out, scale=0.5), normal(rows, n_out)
    args = [t.double() for t in (dy, x, w, b)]
    for name in ref.ACTS if rows * n_in * n_out < 1 << 24 else ["silu"]:
        got = nd.linear_grad(dy, x, w, b, name)
        want = ref.linear_grad(*args, name)[2]
        check(got[2], want, bias_bound(*args, name, kind), name)
        if name != "relu" and n_out >= 1000:        # (relu's slope jumps where z is 0 but for the sum's rounding)
            near(got[2], want, want.to(TYPE[kind]).double(), name)
        alone = nd.linear_grad(dy, x, w, b, name, False, False, True)
        assert torch.equal(alone[2], got[2])


@pytest.mark.parametrize("rows,n_in,n_out", [(300, 64, 96), (300, 1024, 100)])
def test_bias_gradient_of_halves_out_of_their_range(nd, rows, n_in, n_out):
    """dz of halves that is written a second time, with a factor, is not added up a second time."""
    normal = make(6, "f16")
    x, w, b = normal(rows, n_in), normal(n_out, n_in, scale=8.0 * (64 / n_in) ** 0.5), normal(n_out)
    for scale in (2.0 ** -20, 2.0 ** 9):
        dy = (normal(rows, n_out).double() * scale).to(torch.float16)
        args = [t.double() for t in (dy, x, w, b)]
        check(nd.linear_grad(dy, x, w, b, "sigmoid")[2], ref.linear_grad(*args, "sigmoid")[2], bias_bound(*args, "sigmoid", "f16"), scale)

"""The root-mean-square norm where its results lie over its inputs: in place as the interface allows, or refused."""
import pytest

import rms_ref
from encoder_ref import F32
from test_gpu_encoder import KINDS, check, make, values

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
EPS = 1e-3


@pytest.fixture(scope="module")
def nd():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2607_03574_amd as m
    return m


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("n", [130, 1024, 8200, 20001])     # rows in registers of 64 and of 256 threads, and longer ones
def test_norm_updates_a_residual_in_place(nd, kind, n):
    """y and h may be x and residual themselves, either way round."""
    rows, code = 5, {"f32": 0, "bf16": 1, "f16": 2}[kind]
    normal = make(n)
    x, r, w = (normal(*s, kind=kind)[0] for s in ((rows, n), (rows, n), (n,)))
    y, h, rstd = nd.rms_norm(x, w, r, EPS)
    y8, scale, _ = nd.rms_norm_8bit(x, w, r, EPS)
    stream = torch.cuda.current_stream().cuda_stream
    for to_y, to_h in (("new", "x"), ("new", "r"), ("x", "r"), ("r", "x"), ("x", "new"), ("r", "new")):
        t = dict(x=x.clone(), r=r.clone(), new=torch.empty_like(x))
        at_y, at_h = t[to_y], t[to_h]
        found = torch.empty(rows, device="cuda")
        st = nd._rms(code, t["x"].data_ptr(), rows, n, n, t["r"].data_ptr(), n, w.data_ptr(), EPS, at_y.data_ptr(), n,
                     at_h.data_ptr(), n, found.data_ptr(), stream)
        assert st == nd.OK
        assert torch.equal(at_h, h) and torch.equal(at_y, y) and torch.equal(found, rstd), (to_y, to_h)
    for to_h in ("x", "r"):
        t, at, found = dict(x=x.clone(), r=r.clone()), torch.empty_like(y8), torch.empty(rows, device="cuda")
        st = nd._rms_8bit(code, t["x"].data_ptr(), rows, n, n, t["r"].data_ptr(), n, w.data_ptr(), EPS, at.data_ptr(), n,
                          found.data_ptr(), t[to_h].data_ptr(), n, stream)
        assert st == nd.OK
        assert torch.equal(t[to_h], h) and torch.equal(at.view(torch.uint8), y8.view(torch.uint8)) and torch.equal(found, scale), to_h
    # through the binding, which returns h
    t = x.clone()
    y2, h2, _ = nd.rms_norm(t, w, r, EPS, out=t)
    assert y2 is t and torch.equal(t, y) and torch.equal(h2, h)


def test_norm_without_a_residual_refuses_its_input_as_out(nd):
    """h, which the gradient takes, is x there."""
    big = torch.randn(9, 64, device="cuda")
    for x, out in ((big, big), (big[:5], big[4:]), (big[:, :30], big[:, :30])):
        with pytest.raises(ValueError, match="out"):
            nd.rms_norm(x, out=out)
    y, h, _ = nd.rms_norm(big[:4], out=big[4:8])      # apart from it
    check(y, rms_ref.rms(values(h), None, 1e-5)[0], 80 * F32 * abs(values(y)) + 1e-30)

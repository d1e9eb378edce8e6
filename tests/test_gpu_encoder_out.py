"""Results of the encoder block's operators that would lie over their inputs are refused, where other threads still read those."""
import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def nd():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2607_03574_amd as m
    return m


def test_products_and_attention_refuse_their_inputs_as_out(nd):
    x, w, r = (torch.randn(s, 64, device="cuda") for s in (80, 64, 80))
    for a in (x, r):
        for out, inputs in ((a, dict(x=a, weight=w)), (a[:64], dict(x=x[:64].clone(), weight=a[:64]))):
            with pytest.raises(ValueError, match="out"):
                nd.linear(**inputs, out=out)
    # the residual is read where a result is written, by the same thread: few rows, one tile a sum, several workgroups a sum
    for rows, n_in, n_out in ((20, 64, 70), (300, 64, 70), (100, 4000, 130)):
        x2, w2, r2 = torch.randn(rows, n_in, device="cuda"), torch.randn(n_out, n_in, device="cuda"), torch.randn(rows, n_out, device="cuda")
        for kind in (torch.float32, torch.bfloat16):
            a, b, t = x2.to(kind), w2.to(kind), r2.to(kind)
            want = nd.linear(a, b, None, "silu", t)
            assert nd.linear(a, b, None, "silu", t, out=t) is t and torch.equal(t, want)
    x8, s = nd.quantize_rows(x)
    y = torch.empty(80, 64, dtype=torch.bfloat16, device="cuda")
    assert nd.linear_8bit(x8, s, x8[:64], s[:64], out=y) is y
    q, k, v = (torch.randn(2, 40, 3, 16, device="cuda") for _ in range(3))
    g, beta = -torch.rand(2, 40, 3, device="cuda"), torch.rand(2, 40, 3, device="cuda")
    for out in (q, k, v):
        with pytest.raises(ValueError, match="out"):
            nd.delta_attention(q, k, v, g, beta, out=out)
        with pytest.raises(ValueError, match="out"):
            nd.delta_attention_step(q[:, 0], k[:, 0], v[:, 0], g[:, 0], beta[:, 0], torch.zeros(2, 3, 16, 16, device="cuda"), out=out[:, 0])

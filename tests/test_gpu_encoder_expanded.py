"""Autograd functions of the encoder operators on tensors whose rows lie over one another."""
import pytest

from encoder_ref import F32

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def nd():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2607_03574_amd as m
    return m


def test_autograd_of_expanded_rows(nd):
    """One row for all: its gradient is the sum of the rows'."""
    from paper_2607_03574_amd import torch_api
    gen = torch.Generator(device="cuda").manual_seed(4)
    one, x, w, r = (torch.randn(s, generator=gen, device="cuda") for s in ((1, 24), (7, 24), (20, 24), (1, 20)))
    dy = torch.randn(7, 20, generator=gen, device="cuda")
    calls = {"norm of it": lambda t: torch_api.rms_norm(t.expand(7, 24), None, x)[0] @ w.T,
             "norm with it": lambda t: torch_api.rms_norm(x, None, t.expand(7, 24))[0] @ w.T,
             "layer norm": lambda t: torch_api.layer_norm(t.expand(7, 24)) @ w.T,
             "projection": lambda t: torch_api.linear(t.expand(7, 24), w, None, "silu"),
             "gated": lambda t: torch_api.gated_ffn(t.expand(7, 24), w, w)}
    for name, call in calls.items():
        got, want = one.clone().requires_grad_(), one.expand(7, 24).clone().requires_grad_()
        y, z = call(got), call(want)
        assert torch.equal(y, z), name
        (g,), (v,) = torch.autograd.grad((y * dy).sum(), got), torch.autograd.grad((z * dy).sum(), want)
        assert torch.allclose(g, v.sum(0, keepdim=True), rtol=0, atol=8 * F32 * float(v.abs().sum(0).max())), name
    t = r.clone().requires_grad_()
    y = torch_api.linear(x, w, None, "silu", t.expand(7, 20))
    assert torch.equal(y, torch_api.linear(x, w, None, "silu", r.expand(7, 20).contiguous()))
    (g,) = torch.autograd.grad((y * dy).sum(), t)
    assert torch.allclose(g, dy.sum(0, keepdim=True), rtol=0, atol=8 * F32 * float(dy.abs().sum(0).max()))

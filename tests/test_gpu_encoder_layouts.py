"""The differentiable layer norm and feed-forward on tensors whose rows do not lie at one stride, or are not
contiguous: the values and gradients of contiguous ones, in the arguments' own shapes."""
import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def api():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2607_03574_amd import torch_api
    return torch_api


VIEWS = {"transposed": lambda t: t.transpose(0, 1), "apart": lambda t: t[:, ::2], "columns": lambda t: t.permute(2, 1, 0)[:, :, :6],
         "every other value": lambda t: t[..., ::2], "broadcast": lambda t: t[:, :1].expand(-1, 5, -1)}


@pytest.mark.parametrize("view", list(VIEWS))
@pytest.mark.parametrize("op", ["norm", "ffn"])
def test_views(api, view, op):
    gen = torch.Generator(device="cuda").manual_seed(3)
    r = lambda *s: torch.randn(s, generator=gen, device="cuda")
    base = r(6, 4, 10)
    n = VIEWS[view](base).shape[-1]
    wide = [0.3 * r(n, 7), 0.3 * r(n, 7)]
    other = [r(n), r(n)] if op == "norm" else wide

    def run(contiguous):
        leaf, weights = base.clone().requires_grad_(), [t.clone().requires_grad_() for t in other]
        x = VIEWS[view](leaf)
        w = weights if op == "norm" else [t.t() for t in weights]       # weights of transposed layers
        if contiguous:
            x, w = x.contiguous(), [t.contiguous() for t in w]
        y = api.layer_norm(x, *w) if op == "norm" else api.gated_ffn(x, *w)
        assert y.shape[:-1] == x.shape[:-1]
        (y * torch.arange(y.numel(), device="cuda").view(y.shape).cos()).sum().backward()
        return [y.detach(), leaf.grad] + [t.grad for t in weights]

    assert all(torch.equal(a, b) for a, b in zip(run(False), run(True)))


def test_a_value_changed_before_backward_is_noticed(api):
    """Saved as it is or as a copy, a backward pass never mixes old and new values."""
    for view in (lambda t: t, lambda t: t.transpose(0, 1)):
        x, w = torch.randn(4, 3, 8, device="cuda"), torch.ones(8, device="cuda", requires_grad=True)
        want = torch.autograd.grad(api.layer_norm(view(x), w).square().sum(), w)[0]
        y = api.layer_norm(view(x), w).square().sum()
        x.zero_()
        try:
            got = torch.autograd.grad(y, w)[0]
        except RuntimeError as e:
            assert "modified by an inplace operation" in str(e)
        else:
            assert torch.equal(got, want)

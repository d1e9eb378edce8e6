"""Tensors that the encoder operators write through their addresses (a step's states, `out`), as autograd sees
them: a backward pass that saved one does not run on the new values, and no graph loses its tensor."""
import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def nd():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2607_03574_amd as m
    return m


def r(*s):
    return torch.randn(s, device="cuda")


def test_a_saved_state_that_was_stepped(nd):
    from paper_2607_03574_amd import torch_api
    q, state, g = r(2, 9, 2, 8).requires_grad_(), r(2, 2, 8, 8), torch.full((2,), -0.1, device="cuda")
    o, _ = torch_api.linear_attention(q, q, q, g, initial_state=state)
    o.sum().backward(retain_graph=True)
    x = r(2, 2, 8)
    nd.linear_attention_step(x, x, x, g, state)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        o.sum().backward()


@pytest.mark.parametrize("op", ["norm", "attention", "step", "ffn"])
def test_a_saved_tensor_that_was_an_output(nd, op):
    from paper_2607_03574_amd import torch_api
    g = torch.full((2,), -0.1, device="cuda")
    saved = r(3, 2, 16) if op == "step" else r(1, 3, 2, 16) if op == "attention" else r(3, 16)
    w = torch.ones(16, device="cuda", requires_grad=True)
    y = torch_api.layer_norm(saved, w)
    if op == "norm":
        nd.layer_norm(r(3, 16), out=saved)
    elif op == "attention":
        nd.linear_attention(*(r(1, 3, 2, 16) for _ in range(3)), g, out=saved)
    elif op == "step":
        nd.linear_attention_step(*(r(3, 2, 16) for _ in range(3)), g, r(3, 2, 16, 16), out=saved)
    else:
        nd.gated_ffn(r(3, 8), r(16, 8), r(16, 8), out=saved)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.sum().backward()


def test_tensors_of_a_graph_are_not_written(nd):
    g, x = torch.full((2,), -0.1, device="cuda"), r(3, 2, 16)
    state = r(3, 2, 16, 16).requires_grad_()
    before = state.detach().clone()
    with pytest.raises(ValueError):
        nd.linear_attention_step(x, x, x, g, state)
    with pytest.raises(ValueError):
        nd.layer_norm(x, out=(r(3, 2, 16).requires_grad_() * 2))
    assert torch.equal(state, before)
    with torch.no_grad():
        o = nd.linear_attention_step(x, x, x, g, state)
    assert not torch.equal(state, before)
    assert torch.equal(o, nd.linear_attention_step(x, x, x, g, before))

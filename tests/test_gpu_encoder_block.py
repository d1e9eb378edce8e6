"""An encoder block of the operators together, as a model calls them: norms that take the residual's addition, projections with
their epilogue, attention by the gated delta rule.  Its output and gradients against the formulas in 64 bits, a stream that
continues it token by token, a graph of a training step, and the block served in 8 bits."""
import math

import pytest

from test_gpu_capture import replays

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

B, T, WIDTH, H, HK, DK, DV, HIDDEN = 3, 70, 96, 4, 2, 24, 32, 136
# Fourteen operators one after the other, forwards and backwards, each off by at most 2e-6 of its terms in norm, and the
# next ones' gain on it: at most four or so (weights of unit gain, a residual beside each).
NEAR = 14 * 2e-6 * 4


@pytest.fixture(scope="module")
def nd():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2607_03574_amd as m
    return m


def weights(seed, dtype=torch.float32):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    r = lambda *s, scale=1.0, shift=0.0: (torch.randn(s, generator=gen, device="cuda") * scale + shift).to(dtype)
    w = dict(qkv=r(2 * HK * DK + H * DV, WIDTH, scale=WIDTH ** -0.5), gates=r(2 * H, WIDTH, scale=WIDTH ** -0.5), gate_bias=r(2 * H),
             mix=r(WIDTH, H * DV, scale=(H * DV) ** -0.5), up=r(HIDDEN, WIDTH, scale=WIDTH ** -0.5), up_bias=r(HIDDEN, scale=0.3),
             down=r(WIDTH, HIDDEN, scale=HIDDEN ** -0.5), n1=r(WIDTH, scale=0.1, shift=1.0), n2=r(WIDTH, scale=0.1, shift=1.0))
    return w, r


def split(qkv, gates):
    """Queries, keys of length one, values, log decays and betas."""
    q, k, v = (t.unflatten(-1, (-1, d)) for t, d in zip(qkv.split([HK * DK, HK * DK, H * DV], -1), (DK, DK, DV)))
    g, b = gates.split(H, -1)
    return q, torch.nn.functional.normalize(k, dim=-1), v, -torch.nn.functional.softplus(g), torch.sigmoid(b)


def block(api, w, x, before, state=None):
    """x [.., T, WIDTH] and the residual stream before it: (what the block adds, the stream, the state)."""
    y, h = api.rms_norm(x, w["n1"], before)
    o, state = api.delta_attention(*split(api.linear(y, w["qkv"]), api.linear(y, w["gates"], w["gate_bias"])), initial_state=state)
    a = api.linear(o.flatten(-2), w["mix"])
    y, h = api.rms_norm(a, w["n2"], h)
    return api.linear(api.linear(y, w["up"], w["up_bias"], "gelu"), w["down"], residual=h), state


def plain(w, x, before, s0):
    """The formulas, a token after the other."""
    norm = lambda t, n: t / torch.sqrt((t * t).mean(-1, keepdim=True) + 1e-5) * n
    h = x + before
    y = norm(h, w["n1"])
    q, k, v, g, b = split(y @ w["qkv"].T, y @ w["gates"].T + w["gate_bias"])
    q, k = (t.repeat_interleave(H // HK, dim=-2) for t in (q, k))
    S, outs = s0, []
    for t in range(x.shape[1]):
        S = S * torch.exp(g[:, t])[..., None, None]
        u = b[:, t, :, None] * (v[:, t] - (k[:, t, :, :, None] * S).sum(-2))
        S = S + k[:, t, :, :, None] * u[..., None, :]
        outs.append((q[:, t, :, :, None] * S).sum(-2) * DK ** -0.5)
    h = h + torch.stack(outs, 1).flatten(-2) @ w["mix"].T
    return torch.nn.functional.gelu(norm(h, w["n2"]) @ w["up"].T + w["up_bias"]) @ w["down"].T + h, S


def apart(a, b):
    return float((a.double().cpu() - b.double().cpu()).norm() / b.double().cpu().norm())


def test_outputs_and_gradients(nd):
    from paper_2607_03574_amd import torch_api
    w, r = weights(1)
    leaves = dict(w, x=r(B, T, WIDTH), before=r(B, T, WIDTH), s0=r(B, H, DK, DV, scale=DK ** -0.5))
    dy, ds = r(B, T, WIDTH), r(B, H, DK, DV)
    found = []
    for wide in (False, True):
        t = {n: (v.double().cpu() if wide else v.clone()).requires_grad_() for n, v in leaves.items()}
        y, S = plain(t, t["x"], t["before"], t["s0"]) if wide else block(torch_api, t, t["x"], t["before"], t["s0"])
        a, b = (dy.double().cpu(), ds.double().cpu()) if wide else (dy, ds)
        ((y * a).sum() + (S * b).sum()).backward()
        found.append([y.detach(), S.detach()] + [v.grad for v in t.values()])
    for name, a, b in zip(("y", "state", *leaves), *found):
        assert apart(a, b) <= NEAR, (name, apart(a, b))


def test_a_stream_continues_it(nd):
    from paper_2607_03574_amd import torch_api
    w, r = weights(2)
    x, before = r(B, T, WIDTH), r(B, T, WIDTH)
    with torch.no_grad():
        whole, last = block(torch_api, w, x, before)
        _, state = block(torch_api, w, x[:, :40].contiguous(), before[:, :40].contiguous())
        for t in range(40, T):
            y, h, _ = nd.rms_norm(x[:, t], w["n1"], before[:, t])
            o = nd.delta_attention_step(*split(nd.linear(y, w["qkv"]), nd.linear(y, w["gates"], w["gate_bias"])), state)
            y, h, _ = nd.rms_norm(nd.linear(o.flatten(-2), w["mix"]), w["n2"], h)
            z = nd.linear(nd.linear(y, w["up"], w["up_bias"], "gelu"), w["down"], residual=h)
            assert apart(z, whole[:, t]) <= NEAR
    assert apart(state, last) <= NEAR


def test_a_training_step_in_a_graph(nd):
    from paper_2607_03574_amd import torch_api
    w, r = weights(3, torch.bfloat16)
    x, before, dy = (r(B, T, WIDTH) for _ in range(3))
    outs = []

    def call(s):
        with torch.cuda.stream(s):
            t = {n: v.detach().requires_grad_() for n, v in dict(w, x=x, before=before).items()}
            y, last = block(torch_api, t, t["x"], t["before"])
            now = [y.detach(), last.detach(), *torch.autograd.grad((y * dy).sum(), list(t.values()))]
            if not outs:
                outs.extend(torch.empty_like(v) for v in now)
            for a, b in zip(outs, now):
                a.copy_(b)

    call(torch.cuda.current_stream())

    def fresh(i):
        _, other = weights(10 + i, torch.bfloat16)
        return [other(B, T, WIDTH) for _ in range(2)]

    replays(call, [x, before], outs, fresh)


def test_two_streams_at_once(nd):
    """The same block on two streams side by side, each with its own data."""
    from paper_2607_03574_amd import torch_api
    w, r = weights(4)
    data = [(r(B, T, WIDTH), r(B, T, WIDTH)) for _ in range(2)]
    with torch.no_grad():
        want = [block(torch_api, w, *d) for d in data]
        torch.cuda.synchronize()
        sides = [torch.cuda.Stream() for _ in range(2)]
        for _ in range(5):
            got = []
            for d, s in zip(data, sides):
                with torch.cuda.stream(s):
                    got.append(block(torch_api, w, *d))
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for g, v in zip(got, want) for a, b in zip(g, v))


def test_served_in_8_bits(nd):
    """The norm's rows as they come, the weights once: what is left is the rounding of both, seen from the values that the
    8-bit rows stand for."""
    w, r = weights(5, torch.bfloat16)
    x, before = r(B * T, WIDTH), r(B * T, WIDTH)
    up8, up_scale = nd.quantize_rows(w["up"])
    y8, scale, h = nd.rms_norm_8bit(x, w["n2"], before)
    z = nd.linear_8bit(y8, scale, up8, up_scale, w["up_bias"], "gelu")
    y, h16, _ = nd.rms_norm(x, w["n2"], before)
    assert torch.equal(h, h16) and z.dtype == torch.bfloat16
    held, up = y8.double() * scale.double()[:, None], up8.double() * up_scale.double()[:, None]
    want = torch.nn.functional.gelu(held @ up.T + w["up_bias"].double())
    # the result's rounding, and what the instructions' sums of eight products cut (2^-13 of the largest)
    limit = 2.0 ** -8 * want.abs() + 1.13 * 7 * 2.0 ** -13 * (held.abs() @ up.abs().T) + math.ldexp(1.0, -20)
    assert torch.all((z.double() - want).abs() <= limit)
    # a value of a row is off by half a step: 2^-4 of itself, or of what stays normal in e4m3, 2^-6, times the scale
    assert torch.all((held - y.double()).abs() <= (2.0 ** -4 + 2.0 ** -8) * y.double().abs() + 2.0 ** -10 * scale.double()[:, None])

"""Gradient of attention by the gated delta rule, and long sequences that are cut into segments, against references in 64
bits: elementwise within derived bounds and in norm, at the lengths, widths, layouts and values where they can go wrong."""
import numpy as np
import pytest

import delta_ref as ref
from test_gpu_delta import CASES, NAMES, case, near
from test_gpu_capture import replays
from test_gpu_encoder import KINDS, check, slope, values

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

# float gradients: products in three stages, each of which leaves out 2^-21 of a term at most, and sums in float; dg adds up
# terms of both signs
FLOAT = 2e-6
LONG = [([1200], 1, 1, 32, 48), ([900, 20, 0, 1100], 2, 1, 40, 24), ([1537], 2, 2, 128, 128), ([700, 700], 1, 1, 64, 80),
        ([1900, 20, 0, 2100], 2, 1, 40, 24)]


@pytest.fixture(scope="module")
def nd():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2607_03574_amd as m
    return m


def compare(t, bounds, got, kind, what=""):
    host = [t[x][1] for x in NAMES]
    do, s0, ds = t["do"][1], t["s0"][1], t["ds"][1]
    want = ref.attention_grad(do, *host, 0.37, bounds, s0, ds)
    limits = ref.bounds_grad(do, *host, 0.37, bounds, s0, ds, want[:5], kind)
    for name, x, w, limit in zip((*NAMES, "s0"), got, want, limits):
        if x is None:
            assert name == "s0" and s0 is None
            continue
        x = x.reshape(w.shape)
        if limit.ndim > w.ndim:
            limit = limit[..., 0]
        check(x, w, np.broadcast_to(limit, w.shape), what + name)
        if w.size > 500:
            near(x, w, what + name, 2 * FLOAT if name == "g" else FLOAT)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("state", [False, True])
@pytest.mark.parametrize("lens,H,Hk,dk,dv", CASES + LONG)
def test_gradient(nd, kind, state, lens, H, Hk, dk, dv):
    t, bounds = case(len(lens) + dk, kind, lens, H, Hk, dk, dv, state)
    args = [t[x][0] for x in NAMES]
    off = torch.tensor(bounds).cuda()
    got = nd.delta_attention_grad(t["do"][0], *args, offsets=off, scale=0.37, initial_state=t["s0"][0], grad_final_state=t["ds"][0])
    compare(t, bounds, got, kind)
    if len(set(lens)) == 1:     # sequences of one length
        shape = lambda x: x.reshape(len(lens), lens[0], *x.shape[1:])
        got = nd.delta_attention_grad(shape(t["do"][0]), *(shape(x) for x in args), scale=0.37, initial_state=t["s0"][0],
                                      grad_final_state=t["ds"][0])
        compare(t, bounds, got, kind, "equal: ")


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("state", [False, True])
@pytest.mark.parametrize("lens,H,Hk,dk,dv", LONG)
def test_long_sequences(nd, kind, state, lens, H, Hk, dk, dv):
    t, bounds = case(len(lens) + dk, kind, lens, H, Hk, dk, dv, state)
    args, host = [t[x][0] for x in NAMES], [t[x][1] for x in NAMES]
    off = torch.tensor(bounds).cuda()
    o, last = nd.delta_attention(*args, offsets=off, scale=0.37, initial_state=t["s0"][0], final_state=True)
    wo, wl, _, _ = ref.attention(*host, 0.37, bounds, t["s0"][1])
    bo, bl = ref.bounds_forward(*host, 0.37, bounds, t["s0"][1], wo, wl, kind)
    check(o, wo, bo, "o")
    check(last, wl, bl, "state")
    near(o, wo, "o")
    near(last, wl, "state", FLOAT)


@pytest.mark.parametrize("lens", [[70, 41], [1100, 950]])
def test_only_what_is_needed(nd, lens):
    t, bounds = case(2, "bf16", lens, 4, 2, 33, 40, True)
    args = [t["do"][0]] + [t[x][0] for x in NAMES]
    off = torch.tensor(bounds).cuda()
    more = dict(offsets=off, initial_state=t["s0"][0], grad_final_state=t["ds"][0])
    want = nd.delta_attention_grad(*args, **more)
    for need in ((True, False, False, False, False), (False, True, False, False, True), (False, False, True, False, False),
                 (False, False, False, True, False), (False,) * 5):
        got = nd.delta_attention_grad(*args, need=need, **more)
        for x, w, there in zip(got, want, (*need, True)):
            assert torch.equal(x, w) if there else x is None
    assert nd.delta_attention_grad(*args, need=(False,) * 5, offsets=off) == (None,) * 6


def test_strides_and_rows_outside(nd):
    """Tensors that are pieces of others, at odd places, NaN around them; outside the sequences gradients are 0."""
    lens, H, Hk, dk, dv = [37, 70], 4, 2, 33, 41
    for kind in KINDS:
        t, bounds = case(5, kind, lens, H, Hk, dk, dv)
        n, off = sum(lens), torch.tensor(bounds).cuda()

        def inside(x):
            big = torch.full((n + 9, *(s + 3 for s in x.shape[1:])), float("nan"), dtype=x.dtype, device="cuda")
            view = big[(slice(None), *(slice(1, 1 + s) for s in x.shape[1:]))]
            view[4:4 + n] = x
            return view

        names = ("do", *NAMES)
        got = nd.delta_attention_grad(*(inside(t[x][0]) for x in names), offsets=off + 4)
        want = nd.delta_attention_grad(*(t[x][0] for x in names), offsets=off)
        for x, w in zip(got[:5], want[:5]):
            assert torch.equal(x[4:4 + n], w) and torch.all(x[:4] == 0) and torch.all(x[4 + n:] == 0)
        turned = [t[x][0].transpose(0, 1).contiguous().transpose(0, 1) for x in names]
        assert all(torch.equal(x, w) for x, w in zip(nd.delta_attention_grad(*turned, offsets=off)[:5], want[:5]))
        # one row for all tokens
        k, one = t["k"][0][:1].expand(n, -1, -1), [t[x][0] for x in names]
        got = nd.delta_attention_grad(one[0], one[1], k, *one[3:], offsets=off)
        want = nd.delta_attention_grad(one[0], one[1], k.contiguous(), *one[3:], offsets=off)
        assert all(torch.equal(x, w) for x, w in zip(got[:5], want[:5]))


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("lens", [[80, 75], [600, 775]])
def test_values_that_are_not_finite(nd, kind, lens):
    """They reach no other sequence and no other head."""
    H, Hk, dk, dv = 2, 2, 40, 72
    t, bounds = case(9, kind, lens, H, Hk, dk, dv)
    off = torch.tensor(bounds).cuda()
    clean = {x: t[x][0] for x in ("do", *NAMES)}
    want = nd.delta_attention_grad(*clean.values(), offsets=off)
    for at in (0, 17, 31, 63, 79):
        for name in clean:
            bad = dict(clean)
            bad[name] = clean[name].clone()
            spot = bad[name][at, 1] if name in ("g", "beta") else bad[name][at, 1, -1:]
            spot.fill_(float("inf") if name in ("g", "v") else float("nan"))
            got = nd.delta_attention_grad(*bad.values(), offsets=off)
            for x, w in zip(got[:5], want[:5]):
                assert torch.equal(x[:, 0], w[:, 0]) and torch.equal(x[lens[0]:], w[lens[0]:]), (name, at)
            # the gradient of q at a token behind it depends on every k and v before
            if name in ("k", "v"):
                assert not torch.isfinite(got[0][lens[0] - 1, 1]).any(), (name, at)


def test_decays_to_nothing_and_none(nd):
    """A log decay of minus infinity, of the type's lowest value or of zero, and betas of 0 and 1."""
    for kind in KINDS:
        t, bounds = case(11, kind, [200], 2, 1, 48, 64, True)
        g, beta = t["g"][0].clone(), t["beta"][0].clone()
        g[10] = float("-inf")
        g[40] = torch.finfo(g.dtype).min
        g[41:60] = 0
        g[70] = -80
        beta[20:30] = 0
        beta[60:90] = 1
        t["g"], t["beta"] = (g, np.maximum(values(g), -1e4)), (beta, values(beta))
        got = nd.delta_attention_grad(t["do"][0], *(t[x][0] for x in NAMES), offsets=torch.tensor(bounds).cuda(), scale=0.37,
                                      initial_state=t["s0"][0], grad_final_state=t["ds"][0])
        compare(t, bounds, got, kind)
        assert torch.all(got[3][10] == 0) and torch.all(got[3][40] == 0)


def test_the_same_key_again_and_again(nd):
    for kind in KINDS:
        n, dk, dv = 150, 64, 32
        t, bounds = case(13, kind, [n], 1, 1, dk, dv)
        k = torch.zeros_like(t["k"][0])
        k[..., 3] = 1
        g = torch.zeros_like(t["g"][0])
        for b in (1.0, 0.75):
            beta = torch.full_like(t["beta"][0], b)
            now = dict(t, k=(k, values(k)), g=(g, values(g)), beta=(beta, values(beta)))
            got = nd.delta_attention_grad(t["do"][0], *(now[x][0] for x in NAMES), offsets=torch.tensor(bounds).cuda(), scale=0.37)
            want = ref.attention_grad(t["do"][1], *(now[x][1] for x in NAMES), 0.37, bounds)
            limits = ref.bounds_grad(t["do"][1], *(now[x][1] for x in NAMES), 0.37, bounds, None, None, want[:5], kind)
            for name, x, w, limit in zip(NAMES, got, want, limits):
                limit = limit[..., 0] if limit.ndim > w.ndim else limit
                check(x, w, np.broadcast_to(limit, w.shape), name)


def test_nothing_to_do(nd):
    for n in (0, 3):
        z = lambda *s: torch.zeros(n, 0, *s, device="cuda")
        s0, ds = torch.zeros(n, 4, 8, 16, device="cuda"), torch.randn(n, 4, 8, 16, device="cuda")
        *grads, d0 = nd.delta_attention_grad(z(4, 16), z(2, 8), z(2, 8), z(4, 16), z(4), z(4), initial_state=s0, grad_final_state=ds)
        assert [tuple(x.shape) for x in grads] == [(n, 0, 2, 8), (n, 0, 2, 8), (n, 0, 4, 16), (n, 0, 4), (n, 0, 4)]
        assert torch.equal(d0, ds)


@pytest.mark.parametrize("long", [False, True])
def test_against_differences(nd, long):
    from paper_2607_03574_amd import torch_api
    gen = torch.Generator(device="cuda").manual_seed(4)
    r = lambda *s: torch.randn(s, generator=gen, device="cuda")
    n = 1700 if long else 75
    off = torch.tensor([0, 30, 30, n]).cuda()
    unit = lambda x: x / x.norm(dim=-1, keepdim=True)
    tensors = [r(n, 1, 12), unit(r(n, 1, 12)), r(n, 2, 20), -torch.rand(n, 2, generator=gen, device="cuda"),
               torch.rand(n, 2, generator=gen, device="cuda"), r(3, 2, 12, 20)]
    f = lambda q, k, v, g, b, s: list(torch_api.delta_attention(q, k, v, g, b, off, 0.3, s))
    tensors = [t.requires_grad_() for t in tensors]
    outs = f(*tensors)
    weights = [r(*o.shape) for o in outs]
    sum((o * w).sum() for o, w in zip(outs, weights)).backward()
    plain = [t.detach() for t in tensors]
    for i, t in enumerate(tensors):
        d = [r(*x.shape) if j == i else torch.zeros_like(x) for j, x in enumerate(plain)]
        want = float((t.grad.double() * d[i].double()).sum())
        # truncation is of order eps^2 times the third derivative (sums of the same terms), rounding of order 2^-22 / eps
        got = slope(f, plain, d, weights, 2.0 ** -9)
        size = float((t.grad.double() * d[i].double()).norm()) * 10 + abs(want)
        assert abs(got - want) <= 2e-3 * size, (i, got, want, size)


def test_autograd(nd):
    """Views of one product, heads first in memory, an output or a state that nothing uses, a second pass."""
    from paper_2607_03574_amd import torch_api
    gen = torch.Generator(device="cuda").manual_seed(5)
    r = lambda *s: torch.randn(s, generator=gen, device="cuda")
    x, gates, s0 = (0.2 * r(2, 45, 2 * 8 + 2 * 8 + 4 * 16)).requires_grad_(), r(2, 45, 8).requires_grad_(), r(2, 4, 8, 16).requires_grad_()

    def parts(copied):
        q, k, v = (t.unflatten(-1, (-1, w)) for t, w in zip(x.split([16, 16, 64], -1), (8, 8, 16)))
        g, b = -torch.nn.functional.softplus(gates[..., :4]), torch.sigmoid(gates[..., 4:])
        if copied:
            return [t.contiguous() for t in (q, k, v, g, b)]
        return q, k.transpose(2, 3).contiguous().transpose(2, 3), v, g, b

    found = []
    for copied in (False, True):
        o, last = torch_api.delta_attention(*parts(copied), initial_state=s0)
        w = torch.arange(o.numel(), device="cuda").view(o.shape).cos()
        (o * w).sum().backward(retain_graph=True)
        last.square().sum().backward()
        found.append([t.grad.clone() for t in (x, gates, s0)])
        for t in (x, gates, s0):
            t.grad = None
    assert all(torch.equal(a, b) for a, b in zip(*found))
    o, last = torch_api.delta_attention(*parts(True), initial_state=s0)
    first, = torch.autograd.grad(o.sum(), s0, create_graph=True)
    with pytest.raises(RuntimeError):
        first.sum().backward()
    # a state that was stepped on since
    state = s0.detach().clone()
    o, _ = torch_api.delta_attention(*parts(True), initial_state=state)
    nd.delta_attention_step(*(t.detach()[:, 0] for t in parts(True)), state)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        o.sum().backward()


@pytest.mark.parametrize("lens", [[33, 90], [1300, 1040]])
def test_streams_and_graphs(nd, lens):
    t, bounds = case(6, "bf16", lens, 2, 1, 64, 48, True)
    args, off = [t[x][0] for x in NAMES], torch.tensor(bounds).cuda()
    state, one = torch.zeros(2, 2, 64, 48, device="cuda"), [x[:2].clone() for x in args]
    outs = []

    def call(s):
        o, last = nd.delta_attention(*args, offsets=off, initial_state=t["s0"][0], final_state=True, stream=s)
        grads = nd.delta_attention_grad(t["do"][0], *args, offsets=off, initial_state=t["s0"][0], grad_final_state=t["ds"][0], stream=s)
        with torch.cuda.stream(s):
            state.copy_(last)
        step = nd.delta_attention_step(*one, state, stream=s)
        with torch.cuda.stream(s):
            now = [o, last, *grads, state, step]
            if not outs:
                outs.extend(torch.empty_like(x) for x in now)
            for a, b in zip(outs, now):
                a.copy_(b)

    call(torch.cuda.current_stream())

    def fresh(i):
        other, _ = case(20 + i, "bf16", lens, 2, 1, 64, 48, True)
        return [other[x][0] for x in NAMES]

    replays(call, args, outs, fresh)


def test_refusals(nd):
    t, bounds = case(1, "f32", [5, 4], 4, 2, 8, 8)
    q, k, v, g, b, do = (t[x][0] for x in (*NAMES, "do"))
    off = torch.tensor(bounds).cuda()
    for bad in (dict(q=q[:, :1].expand(-1, 3, -1)), dict(k=k[:4]), dict(g=g[:, :3]), dict(beta=b[:8]), dict(do=do[..., :7])):
        with pytest.raises((ValueError, nd.NdvmError)):
            nd.delta_attention_grad(**{**dict(do=do, q=q, k=k, v=v, g=g, beta=b, offsets=off), **bad})
    for bad in (dict(g=g.bfloat16()), dict(beta=b.double()), dict(do=do.half())):
        with pytest.raises(TypeError):
            nd.delta_attention_grad(**{**dict(do=do, q=q, k=k, v=v, g=g, beta=b, offsets=off), **bad})
    with pytest.raises(ValueError):
        nd.delta_attention_grad(do, q, k, v, g, b, off, initial_state=torch.zeros(2, 4, 8, 9, device="cuda"))
    with pytest.raises(ValueError):
        nd.delta_attention(q[None], k[None], v[None], g[None], b[None], off)
    with pytest.raises(nd.NdvmError):
        nd.delta_attention(q, k, v, g, b, off, scale=float("inf"))
    wide = torch.zeros(9, 2, 257, device="cuda")
    with pytest.raises(nd.NdvmError) as e:
        nd.delta_attention(wide, wide, v, g, b, off)
    assert e.value.status == nd.E_UNSUPPORTED
    with pytest.raises(nd.NdvmError):
        nd.delta_attention_step(q, k, v, g, b, torch.zeros(8, 4, 8, 8, device="cuda"))      # 9 streams, 8 slots


def test_places_beyond_32_bits(nd):
    """Rows 16 MB apart, in 5 GB, and states in slots of 4.4 GB: the same bits as side by side."""
    n, d = 300, 16
    t, bounds = case(21, "bf16", [n], 1, 1, d, d)
    off, big = torch.tensor(bounds).cuda(), torch.empty(n, 1 << 23, dtype=torch.bfloat16, device="cuda")

    def far(x, at):
        view = big[:, at:at + x[0].numel()].view(x.shape)
        view.copy_(x)
        return view

    near_by = [t[x][0] for x in ("do", *NAMES)]
    apart = [far(x, 16 * i) for i, x in enumerate(near_by)]
    assert apart[0].stride(0) == 1 << 23
    out = big[:, 200:200 + d].view(n, 1, d)
    o, last = nd.delta_attention(*apart[1:], offsets=off, out=out, final_state=True)
    want = nd.delta_attention(*near_by[1:], offsets=off, final_state=True)
    assert torch.equal(o, want[0]) and torch.equal(last, want[1])
    got, want = (nd.delta_attention_grad(*x, offsets=off) for x in (apart, near_by))
    assert all(torch.equal(a, b) for a, b in zip(got[:5], want[:5]))
    del big, apart, out, o
    t, _ = case(22, "bf16", [1, 1], 16, 16, 128, 128, True)
    args, s0 = [t[x][0] for x in NAMES], t["s0"][0]
    state = torch.empty(4200, 16, 128, 128, device="cuda")
    slots = torch.tensor([0, 4199], device="cuda")
    state[slots] = s0
    small = s0.clone()
    assert torch.equal(nd.delta_attention_step(*args, state, slots=slots), nd.delta_attention_step(*args, small))
    assert torch.equal(state[slots], small)

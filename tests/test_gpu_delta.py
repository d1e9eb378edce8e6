"""Attention by the gated delta rule, its single-token step and its gradient, against references in 64 bits: elementwise
within derived bounds and in norm, at the lengths, widths, layouts and values where they can go wrong."""
import numpy as np
import pytest

import delta_ref as ref
from encoder_ref import F32, UNIT
from test_gpu_encoder import KINDS, TYPE, check, make, values

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

# tokens of the sequences, heads, heads of q and k, dk, dv
CASES = [([1], 1, 1, 1, 1), ([0, 1, 2], 2, 1, 16, 16), ([15, 16, 17], 2, 2, 33, 20), ([31, 32, 33], 2, 1, 20, 33),
         ([63, 0, 65, 64], 4, 2, 64, 64), ([130, 31, 1, 33], 3, 1, 40, 72), ([97, 200], 2, 2, 128, 128), ([70, 12], 2, 1, 128, 64),
         ([40, 33], 1, 1, 200, 150), ([5], 1, 1, 256, 256), ([301], 1, 1, 64, 128), ([129, 128], 4, 4, 32, 40)]


@pytest.fixture(scope="module")
def nd():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2607_03574_amd as m
    return m


def case(seed, kind, lens, H, Hk, dk, dv, state=False):
    """Keys of length one at most, betas between 0 and 1, decays from none to strong ones."""
    rng = np.random.default_rng(seed)
    n = sum(lens)

    def made(x):
        t = torch.tensor(x).to(TYPE[kind]).cuda()
        return t, values(t)

    def unit(*shape):
        x = rng.normal(size=shape) + 0.3
        return x / np.sqrt((x ** 2).sum(-1, keepdims=True)) * 0.99

    t = dict(q=made(unit(n, Hk, dk) * 2.0), k=made(unit(n, Hk, dk)), v=made(rng.normal(size=(n, H, dv))),
             g=made(-np.exp2(rng.uniform(-9, 1, (n, H)))), beta=made(rng.uniform(0, 1, (n, H)) ** 0.5), do=made(rng.normal(size=(n, H, dv))))
    bounds = np.concatenate([[0], np.cumsum(lens)]).astype(np.int64)
    for name in ("s0", "ds"):
        x = torch.tensor(rng.normal(size=(len(lens), H, dk, dv)) / dk ** 0.5).float().cuda() if state else None
        t[name] = (x, None if x is None else values(x))
    return t, bounds


def near(got, want, what="", f32=1e-6):
    """In norm: float sums lose some 2^-24 of their terms on average, and a 16-bit result its own rounding."""
    rounded = values(torch.tensor(want).to(got.dtype))
    norm = np.linalg.norm(want)
    limit = f32 * norm if got.dtype == torch.float32 else 1.05 * np.linalg.norm(rounded - want) + 1e-6 * norm
    off = np.linalg.norm(values(got) - want)
    assert off <= limit + 1e-30, (what, off / max(norm, 1e-300), limit / max(norm, 1e-300))


NAMES = ("q", "k", "v", "g", "beta")


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("state", [False, True])
@pytest.mark.parametrize("lens,H,Hk,dk,dv", CASES)
def test_delta_attention(nd, kind, state, lens, H, Hk, dk, dv):
    t, bounds = case(len(lens) + dk, kind, lens, H, Hk, dk, dv, state)
    args, host = [t[x][0] for x in NAMES], [t[x][1] for x in NAMES]
    s0, sv = t["s0"]
    off = torch.tensor(bounds).cuda()
    o, last = nd.delta_attention(*args, offsets=off, scale=0.37, initial_state=s0, final_state=True)
    wo, wl, _, _ = ref.attention(*host, 0.37, bounds, sv)
    bo, bl = ref.bounds_forward(*host, 0.37, bounds, sv, wo, wl, kind)
    check(o, wo, bo, "o")
    check(last, wl, bl, "state")
    if wo.size > 500:
        near(o, wo, "o")
        near(last, wl, "state")
    if len(set(lens)) == 1:     # the same as sequences of one length, with no state kept
        shape = lambda x: x.reshape(len(lens), lens[0], *x.shape[1:])
        o2, none = nd.delta_attention(*(shape(x) for x in args), scale=0.37, initial_state=s0)
        assert none is None
        check(o2.reshape(o.shape), wo, bo)


def test_sequences_of_one_length_and_a_default_scale(nd):
    t, bounds = case(3, "bf16", [45] * 6, 4, 2, 24, 48, True)
    args, host = [t[x][0] for x in NAMES], [t[x][1] for x in NAMES]
    shape = lambda x: x.reshape(6, 45, *x.shape[1:])
    o, last = nd.delta_attention(*(shape(x) for x in args), initial_state=t["s0"][0], final_state=True)
    packed = nd.delta_attention(*args, offsets=torch.tensor(bounds).cuda(), initial_state=t["s0"][0], final_state=True)
    assert torch.equal(o.reshape(packed[0].shape), packed[0]) and torch.equal(last, packed[1])
    wo, wl, _, _ = ref.attention(*host, 24 ** -0.5, bounds, t["s0"][1])
    near(o.reshape(270, 4, 48), wo)
    near(last, wl)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("slots", [False, True])
@pytest.mark.parametrize("n,H,Hk,dk,dv", [(1, 1, 1, 1, 1), (3, 4, 2, 33, 20), (5, 2, 2, 128, 128), (9, 3, 1, 100, 77), (2, 2, 1, 256, 200),
                                         (200, 16, 4, 64, 128), (260, 16, 16, 128, 128)])
def test_step(nd, kind, slots, n, H, Hk, dk, dv):
    t, _ = case(n + dk, kind, [1] * n, H, Hk, dk, dv)
    args, host = [t[x][0] for x in NAMES], [t[x][1] for x in NAMES]
    rng = np.random.default_rng(n)
    m = n + 3 if slots else n
    state = torch.tensor(rng.normal(size=(m, H, dk, dv)) / dk ** 0.5).float().cuda()
    at = rng.permutation(m)[:n]
    if slots and n > 4:
        at[2], at[4] = -1, m + 5        # streams without a state
    before, there = values(state), (at >= 0) & (at < m) if slots else np.ones(n, bool)
    where = np.where(there, at, 0) if slots else np.arange(n)
    o = nd.delta_attention_step(*args, state, slots=torch.tensor(at).cuda() if slots else None, scale=0.37)
    wo, wl, _, _ = ref.attention(*host, 0.37, np.arange(n + 1), before[where])
    bo, bl = ref.bounds_forward(*host, 0.37, np.arange(n + 1), before[where], wo, wl, kind)
    wo[~there], bo[~there] = 0, 0
    check(o, wo, bo, "o")
    want, bound = before.copy(), np.zeros_like(before)
    want[where[there]], bound[where[there]] = wl[there], bl[there]
    check(state, want, bound, "state")      # the slots of no stream keep their bits


def test_streams_continue_a_sequence(nd):
    """Half a sequence at once and the rest token by token is the whole sequence; so are two halves at once."""
    for kind in KINDS:
        t, bounds = case(8, kind, [90, 90], 4, 2, 64, 96, True)
        shape = lambda x: x.reshape(2, 90, *x.shape[1:])
        args, s0 = [shape(t[x][0]) for x in NAMES], t["s0"][0]
        o, last = nd.delta_attention(*args, initial_state=s0, final_state=True)
        a, state = nd.delta_attention(*(x[:, :47] for x in args), initial_state=s0, final_state=True)
        b, end = nd.delta_attention(*(x[:, 47:] for x in args), initial_state=state, final_state=True)
        host = [t[x][1] for x in NAMES]
        wo, wl, _, _ = ref.attention(*host, 64 ** -0.5, bounds, t["s0"][1])
        near(torch.cat([a, b], 1).reshape(180, 4, 96), wo)
        near(end, wl)
        steps = [nd.delta_attention_step(*(x[:, i] for x in args), state) for i in range(47, 90)]
        near(torch.cat([a, torch.stack(steps, 1)], 1).reshape(180, 4, 96), wo)
        near(state, wl)
        assert torch.equal(last, nd.delta_attention(*args, initial_state=s0, final_state=True)[1])


def test_strides_alignment_and_rows_outside(nd):
    """Tensors that are pieces of others, at odd places; tokens in front of the first sequence and behind the last are
    left as they were."""
    lens, H, Hk, dk, dv = [37, 70], 4, 2, 33, 41
    for kind in KINDS:
        t, bounds = case(5, kind, lens, H, Hk, dk, dv)
        n = sum(lens)
        rng = np.random.default_rng(1)

        def inside(x, pad):     # a piece of a larger tensor whose other places are NaN
            big = torch.full((n + 9, *(s + p for s, p in zip(x.shape[1:], pad))), float("nan"), dtype=x.dtype, device="cuda")
            view = big[tuple([slice(4, 4 + n)] + [slice(p - p // 2, p - p // 2 + s) for s, p in zip(x.shape[1:], pad)])]
            view.copy_(x)
            return big[tuple([slice(None)] + [slice(p - p // 2, p - p // 2 + s) for s, p in zip(x.shape[1:], pad)])]

        args = [inside(t[x][0], (1, 3) if x in "qkv" else (3,)) for x in NAMES]
        out = torch.full((n + 9, H, dv + 5), -7.25, dtype=TYPE[kind], device="cuda")
        o, last = nd.delta_attention(*args, offsets=torch.tensor(bounds + 4).cuda(), out=out[:, :, 3:3 + dv], final_state=True)
        want = nd.delta_attention(*(t[x][0] for x in NAMES), offsets=torch.tensor(bounds).cuda(), final_state=True)
        assert torch.equal(o[4:4 + n], want[0]) and torch.equal(last, want[1])
        assert torch.all(out[:4] == -7.25) and torch.all(out[4 + n:] == -7.25) and torch.all(out[:, :, :3] == -7.25) and torch.all(out[:, :, 3 + dv:] == -7.25)
        # heads first in memory
        turned = [t[x][0].transpose(0, 1).contiguous().transpose(0, 1) for x in NAMES]
        assert torch.equal(nd.delta_attention(*turned, offsets=torch.tensor(bounds).cuda())[0], want[0])


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("dk,dv", [(128, 64), (64, 40), (24, 130)])
def test_values_that_are_not_finite(nd, kind, dk, dv):
    """They reach no earlier token, no other column, head or sequence."""
    lens, H, Hk = [80, 75], 2, 2
    t, bounds = case(9, kind, lens, H, Hk, dk, dv)
    off = torch.tensor(bounds).cuda()
    clean = {x: t[x][0] for x in NAMES}
    o, last = nd.delta_attention(*clean.values(), offsets=off, final_state=True)
    for at in (0, 17, 31, 32, 50, 79):
        for name in NAMES:
            bad = dict(clean)
            bad[name] = clean[name].clone()
            spot = bad[name][at, 1] if name in ("g", "beta") else bad[name][at, 1, -1:]
            spot.fill_(float("inf") if name in ("g", "v") else float("nan"))
            z, end = nd.delta_attention(*bad.values(), offsets=off, final_state=True)
            hit = torch.zeros_like(z, dtype=torch.bool)
            hit_end = torch.zeros_like(end, dtype=torch.bool)
            if name == "q":
                hit[at, 1] = True
            elif name == "v":
                hit[at:80, 1, -1] = True
                hit_end[0, 1, :, -1] = True
            else:
                hit[at:80, 1] = True
                hit_end[0, 1] = True
            assert not torch.isfinite(z[hit]).any() and torch.equal(z[~hit], o[~hit]), (at, name)
            assert not torch.isfinite(end[hit_end]).any() and torch.equal(end[~hit_end], last[~hit_end]), (at, name)


def test_decays_to_nothing_and_none(nd):
    """A log decay of minus infinity, of the type's lowest value or of zero, and betas of 0 and 1."""
    for kind in KINDS:
        t, bounds = case(11, kind, [100], 2, 1, 48, 64, True)
        g, beta = t["g"][0].clone(), t["beta"][0].clone()
        g[10] = float("-inf")
        g[40] = torch.finfo(g.dtype).min
        g[41:60] = 0
        beta[20:30] = 0
        beta[60:90] = 1
        gv = values(g)
        args = [t["q"][0], t["k"][0], t["v"][0], g, beta]
        host = [values(x) for x in args]
        host[3] = np.maximum(gv, -1e4)
        o, last = nd.delta_attention(*args, offsets=torch.tensor(bounds).cuda(), initial_state=t["s0"][0], scale=1.0, final_state=True)
        wo, wl, _, _ = ref.attention(*host, 1.0, bounds, t["s0"][1])
        near(o, wo)
        near(last, wl)


def test_the_same_key_again_and_again(nd):
    """Keys that are all alike: the inverse of a chunk has its largest entries; with beta 1 the state holds the last value."""
    for kind in KINDS:
        n, dk, dv = 100, 64, 32
        k = torch.zeros(1, n, 1, dk, device="cuda", dtype=TYPE[kind])
        k[..., 3] = 1
        v = torch.randn(1, n, 1, dv, generator=torch.Generator(device="cuda").manual_seed(1), device="cuda").to(TYPE[kind])
        one, zero = torch.ones(1, n, 1, device="cuda", dtype=TYPE[kind]), torch.zeros(1, n, 1, device="cuda", dtype=TYPE[kind])
        o, last = nd.delta_attention(k, k, v, zero, one, scale=1.0, final_state=True)
        assert torch.allclose(o.double(), v.double(), rtol=UNIT[kind] + 64 * F32, atol=200 * F32)
        assert torch.allclose(last[0, 0, 3].double(), v[0, -1, 0].double(), rtol=0, atol=200 * F32)
        host = [values(x[0]) for x in (k, k, v, zero, one * 0.75)]
        o, last = nd.delta_attention(k, k, v, zero, one * 0.75, scale=1.0, final_state=True)
        wo, wl, _, _ = ref.attention(*host, 1.0, [0, n])
        near(o[0], wo)
        near(last, wl)


def test_nothing_to_do(nd):
    for n in (0, 3):
        z = lambda *s: torch.zeros(n, 0, *s, device="cuda")
        o, last = nd.delta_attention(z(2, 8), z(2, 8), z(4, 16), z(4), z(4), final_state=True)
        assert o.shape == (n, 0, 4, 16) and last.shape == (n, 4, 8, 16) and torch.all(last == 0)
    s0 = torch.randn(2, 4, 8, 16, device="cuda")
    e = lambda *s: torch.zeros(0, *s, device="cuda")
    o, last = nd.delta_attention(e(2, 8), e(2, 8), e(4, 16), e(4), e(4), offsets=torch.zeros(3, dtype=torch.int64, device="cuda"),
                                 initial_state=s0, final_state=True)
    assert o.shape == (0, 4, 16) and torch.equal(last, s0)

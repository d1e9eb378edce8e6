"""Heads of more than 128 widths in sequences that are cut into segments, by the gated delta rule and its gradient."""
import pytest

import delta_ref as ref
from delta_wide_sizes import WIDE
from test_gpu_delta import NAMES, case, near
from test_gpu_delta_grad import FLOAT, compare
from test_gpu_encoder import KINDS, check

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def nd():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2607_03574_amd as m
    return m


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("state", [False, True])
@pytest.mark.parametrize("lens,H,Hk,dk,dv", WIDE)
def test_wide_heads_of_long_sequences(nd, kind, state, lens, H, Hk, dk, dv):
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
    got = nd.delta_attention_grad(t["do"][0], *args, offsets=off, scale=0.37, initial_state=t["s0"][0], grad_final_state=t["ds"][0])
    compare(t, bounds, got, kind)
    if len(lens) == 1:      # the same sequence without offsets
        one = [x[None] for x in args]
        o2, last2 = nd.delta_attention(*one, scale=0.37, initial_state=t["s0"][0], final_state=True)
        check(o2[0], wo, bo, "o, equal lengths")
        check(last2, wl, bl, "state, equal lengths")
        got = nd.delta_attention_grad(t["do"][0][None], *one, scale=0.37, initial_state=t["s0"][0], grad_final_state=t["ds"][0])
        compare(t, bounds, got, kind, "equal: ")


@pytest.mark.parametrize("kind", KINDS)
def test_values_that_are_not_finite_in_wide_heads(nd, kind):
    """From a key or gate that is not finite on its head is NaN, over all segments that follow; a value of v only its column."""
    lens, H, Hk, dk, dv = WIDE[1]
    t, bounds = case(8, kind, lens, H, Hk, dk, dv)
    args, off = [t[x][0] for x in NAMES], torch.tensor(bounds).cuda()
    o, last = nd.delta_attention(*args, offsets=off, final_state=True)
    for which in (1, 2, 4):
        at, bad = 300, [x.clone() for x in args]
        bad[which][at, 0] = float("nan") if which != 2 else bad[2][at, 0]
        if which == 2:
            bad[2][at, 0, 5] = float("inf")
        p, end = nd.delta_attention(*bad, offsets=off, final_state=True)
        hit = torch.zeros_like(p, dtype=torch.bool)
        gone = slice(0, H // Hk if which == 1 else 1)     # heads that read that key
        if which == 2:
            hit[at:lens[0], 0, 5] = True
        else:
            hit[at:lens[0], gone] = True
        assert torch.isnan(p[hit]).all() and torch.equal(p[~hit], o[~hit]), which
        if which == 2:
            assert torch.isnan(end[0, 0, :, 5]).all() and torch.isfinite(end).sum() == end.numel() - dk
        else:
            assert torch.isnan(end[0, gone]).all() and torch.equal(end[1:], last[1:])

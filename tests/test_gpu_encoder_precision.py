"""How many bits the encoder operators keep: norm-wise errors against 64 bits.

The elementwise bounds of encoder_ref hold for sums that lose as much as they can; these
limits are near what the kernels' arithmetic gives for the sums of random terms, so that a
part of an operand that was left out would show.

16-bit results: one rounding of the exact value is off by r, measured here by rounding the 64-bit
result.  Operands of at least 16 bits on the way (errors below 2^-16 of each term, of either sign) add
less than 0.3 r in norm, even where they add up over terms, so the error is within sqrt(1 + 0.3^2) r
< 1.05 r.  One more rounding to the type's bits on the way would make it sqrt(2) r.

float results: products of parts leave out at most 2^-21 of a term, 2^-24 on average, and float sums of some
hundred steps 2^-24 times the root of their number: 3e-7 to 5e-7, the limit twice that.  Without the third
part of an operand the error is 2^-16 or so, fifteen times the limit.
"""
import numpy as np
import pytest

import encoder_ref as ref

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

TYPE = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
KINDS = ["f32", "bf16", "f16"]
ONCE = 1.05         # roundings of a 16-bit result
FLOAT = 1e-6


@pytest.fixture(scope="module")
def nd():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2607_03574_amd as m
    return m


def make(seed):
    rng = np.random.default_rng(seed)

    def normal(*shape, kind="f32", scale=1.0):
        t = torch.tensor(rng.normal(size=shape) * scale).to(TYPE[kind]).cuda()
        return t, values(t)

    return normal


def values(t):
    return t.detach().double().cpu().numpy()


def close(got, want, kind, what, once=ONCE):
    size = np.linalg.norm(want)
    error = np.linalg.norm(values(got) - want) / size
    if got.dtype == torch.float32:
        limit = FLOAT
    else:
        limit = once * np.linalg.norm(values(torch.tensor(want).to(got.dtype)) - want) / size
    assert error <= limit, (what, kind, error, limit)


# tokens of the sequences, heads, kv heads, dk, dv: every width the kernels are built for, whole and cut
SIZES = [([90], 2, 2, 64, 64), ([300, 70], 2, 1, 64, 128), ([400], 2, 2, 128, 64), ([33, 500], 2, 1, 128, 128), ([60, 41], 2, 1, 40, 72),
         ([70], 1, 1, 200, 150)]


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("aligned", [True, False])
@pytest.mark.parametrize("lens,H,Hk,dk,dv", SIZES)
def test_linear_attention(nd, kind, aligned, lens, H, Hk, dk, dv):
    normal = make(dk + dv)
    n = sum(lens)

    def tensor(*shape):
        t, v = normal(*shape, kind=kind)
        if not aligned:
            t = torch.empty(t.numel() + 1, dtype=t.dtype, device="cuda")[1:].view(t.shape).copy_(t)
        return t, v

    (q, qv), (k, kv), (v, vv), (do, dov) = tensor(n, H, dk), tensor(n, Hk, dk), tensor(n, Hk, dv), tensor(n, H, dv)
    (s0, s0v), (ds, dsv) = normal(len(lens), H, dk, dv, scale=4.0), normal(len(lens), H, dk, dv, scale=4.0)
    g = torch.tensor([-0.02 / 4.0 ** h for h in range(H)], dtype=torch.float32).cuda()
    bounds = np.concatenate([[0], np.cumsum(lens)]).astype(np.int64)
    off = torch.tensor(bounds).cuda()
    o, last = nd.linear_attention(q, k, v, g, offsets=off, scale=0.3, initial_state=s0, final_state=True)
    wo, wl = ref.attention(qv, kv, vv, values(g), 0.3, bounds, s0v)
    close(o, wo, kind, "o")
    close(last, wl, kind, "state")
    got = nd.linear_attention_grad(do, q, k, v, g, offsets=off, scale=0.3, initial_state=s0, grad_final_state=ds)
    want = ref.attention_grad(dov, qv, kv, vv, values(g), 0.3, bounds, s0v, dsv)
    for a, b, what in zip(got, want, ("dq", "dk", "dv", "d s0")):
        close(a, b, kind, what)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("rows,n_in,n_out", [(40, 300, 200), (130, 264, 200), (700, 200, 1000), (70, 2100, 100)])
def test_gated_ffn(nd, kind, rows, n_in, n_out):
    normal = make(rows)
    (x, xv), (dh, dhv) = normal(rows, n_in, kind=kind), normal(rows, n_out, kind=kind)
    (wg, wgv), (wu, wuv) = (normal(n_out, n_in, kind=kind, scale=n_in ** -0.5) for _ in range(2))
    close(nd.gated_ffn(x, wg, wu), ref.ffn(xv, wgv, wuv, "silu"), kind, "h")
    for a, b, what in zip(nd.gated_ffn_grad(dh, x, wg, wu), ref.ffn_grad(dhv, xv, wgv, wuv, "silu"), ("dx", "dw_gate", "dw_up")):
        # dg and du are rounded to the type, as operands: two roundings of one size, sqrt(2)
        close(a, b, kind, what, once=1.5)


@pytest.mark.parametrize("rows,n_in,n_out", [(7020, 1036, 423), (1289, 2668, 1028)])
def test_float_ffn_of_long_sums(nd, rows, n_in, n_out):
    """Sums that one workgroup forms whole, over six products of parts."""
    normal = make(n_in)
    (x, xv), (wg, wgv), (wu, wuv) = normal(rows, n_in), normal(n_out, n_in, scale=n_in ** -0.5), normal(n_out, n_in, scale=n_in ** -0.5)
    close(nd.gated_ffn(x, wg, wu), ref.ffn(xv, wgv, wuv, "silu"), "f32", "h")


# ---------------------------------------------------------------- float: all 24 bits of an operand
FINE = 1.0 + 2.0 ** -12 + 2.0 ** -20        # a value in each of its three parts
REST = 2.0 ** -12 + 2.0 ** -20              # what is left where the leading part cancels


@pytest.mark.parametrize("rows", [5, 100])      # few rows have a kernel of their own
def test_float_ffn_keeps_the_lower_parts(nd, rows):
    """Leading parts cancel; what is left is a sum of powers of two that float holds exactly."""
    n_in, n_out = 96, 40
    fine = torch.full((n_in,), 1.0)
    fine[::2] = FINE
    sign = torch.ones(n_in)
    sign[1::2] = -1.0
    first = torch.zeros(n_in)
    first[0] = 1.0
    for x, w in ((fine, sign), (sign, fine)):       # in either operand
        x, w, up = (t.cuda() for t in (x.repeat(rows, 1), w.repeat(n_out, 1), first.repeat(n_out, 1)))
        u = float(x[0, 0])
        h = values(nd.gated_ffn(x, w, up, "relu"))
        want = n_in // 2 * REST * u
        assert np.all(np.abs(h - want) <= 2.0 ** -23 * want), (h[0, 0], want)


@pytest.mark.parametrize("d", [64, 128])
def test_float_attention_keeps_the_lower_parts(nd, d):
    fine, sign, zero = torch.full((d,), 1.0), torch.ones(d), torch.zeros(d)
    fine[::2] = FINE
    sign[1::2] = -1.0
    g = torch.zeros(1, device="cuda")
    left = d // 2 * REST

    def run(q, k, v, s0=None):
        q, k, v = (t.cuda().view(1, 1, 1, d) for t in (q, k, v))
        s0 = s0 if s0 is None else s0.cuda().view(1, 1, d, d)
        return nd.linear_attention(q, k, v, g, scale=1.0, initial_state=s0, final_state=True)

    one = torch.zeros(d)
    one[3] = 1.0
    for q, k in ((fine, sign), (sign, fine)):       # a pair's product
        o = run(q, k, torch.ones(d))[0]
        assert torch.all(o == left)
    o, last = run(one, one, fine)                   # what it is multiplied with, and the state's term
    assert torch.equal(o.cpu().view(d), fine) and torch.equal(last[0, 0, 3].cpu(), fine)
    for q, s in ((fine, sign), (sign, fine)):       # what is read from the state
        o = run(q, zero, zero, s[:, None].repeat(1, d))[0]
        assert torch.all(o == left)

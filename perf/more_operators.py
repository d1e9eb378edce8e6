"""More operators of the sequence encoder, as timed cases: attention by the gated delta rule, projections with bias,
activation and residual (also of 8-bit operands), and the root-mean-square norm that takes the residual's addition with
it (also with an 8-bit result).

`run` computes them in plain torch operations in 32 bits (the triangular inverse of the delta rule in 64), or, with `own`
set, through this package's entry points.  Sizes run from one token of a stream to training batches and long
observation series.
"""
import math

import torch

own = False

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SIZE = {"f32": 4, "bf16": 2, "f16": 2}
E4M3 = torch.float8_e4m3fn
CHUNK = 64      # tokens per block of the plain chunked delta rule


# ------------------------------------------------------------------ cases
def listed():
    return [
        # one long series read at once, the state kept for the stream that follows
        dict(name="delta_long", op="delta", type="bf16", seqs=1, tokens=16384, heads=16, qk_heads=16, dk=128, dv=128,
             packed=False, state=False),
        # 37 series of different lengths in one pass, four value heads sharing a key
        dict(name="delta_packed", op="delta", type="bf16", seqs=37, tokens=9001, heads=16, qk_heads=4, dk=64, dv=128,
             packed=True, state=False),
        # the gradient in a training step
        dict(name="delta_grad_batch", op="delta_grad", type="bf16", seqs=8, tokens=16384, heads=16, qk_heads=16, dk=128,
             dv=128, packed=False, state=False),
        # a small model in single precision, series cut in pieces: states go in and their gradients come out
        dict(name="delta_grad_odd", op="delta_grad", type="f32", seqs=3, tokens=2331, heads=6, qk_heads=2, dk=40, dv=72,
             packed=False, state=True),
        # one new point of 192 streams that live in 256 slots
        dict(name="delta_step", op="delta_step", type="bf16", seqs=192, slots=256, heads=16, qk_heads=16, dk=128, dv=128),
        # the way back from a feed-forward for one point of 17 streams: weights are what is read
        dict(name="linear_few", op="linear", type="bf16", rows=17, n_in=4096, n_out=1024, act="none", bias=False,
             residual=True),
        # a projection of a batch, with everything that its epilogue takes
        dict(name="linear_batch", op="linear", type="bf16", rows=8192, n_in=2048, n_out=2048, act="gelu", bias=True,
             residual=True),
        # its gradient in a training step
        dict(name="linear_grad_batch", op="linear_grad", type="bf16", rows=4096, n_in=1024, n_out=4096, act="silu",
             bias=True, residual=False),
        # the batch once more, in 8 bits, as a model that is no longer trained is served
        dict(name="linear_8bit_batch", op="linear_8bit", type="bf16", rows=8192, n_in=2048, n_out=8192, act="gelu",
             bias=True, residual=False),
        # one token of four streams: what a norm costs between two steps of a stream
        dict(name="rms_token", op="rms", type="bf16", rows=4, n=1024, residual=True),
        # the norm's gradient in a training step, joined with what comes back along the residual
        dict(name="rms_grad_batch", op="rms_grad", type="bf16", rows=16384, n=2048, residual=True),
        # the norm in front of an 8-bit projection, 16 series of 2048 points at once
        dict(name="rms_8bit_batch", op="rms_8bit", type="bf16", rows=32768, n=2048, residual=True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["delta", "delta", "delta_grad", "delta_step", "linear", "linear_grad", "linear_8bit", "rms", "rms_grad",
                     "rms_8bit"])
    t = rng.choice(["bf16", "bf16", "bf16", "f16", "f16" if op.endswith("8bit") else "f32"])     # 8 bits stand for 16
    if op.startswith("rms"):
        n = _log(rng, 17, 8192)
        return dict(op=op, type=t, rows=_log(rng, 1, min(32768, (1 << 26) // n)), n=n, residual=rng.random() < 0.7)
    if op.startswith("linear"):
        n_in, n_out = _log(rng, 48, 2048), _log(rng, 48, 8192)
        if op == "linear" and rng.random() < 0.5:
            n_in, n_out = n_out, n_in
        if rng.random() < 0.5:      # widths of most models are multiples of 64
            n_in, n_out = max(64, n_in // 64 * 64), max(64, n_out // 64 * 64)
        rows = _log(rng, 1, 2048 if t == "f32" else 4096 if op == "linear_grad" else 8192)
        return dict(op=op, type=t, rows=rows, n_in=n_in, n_out=n_out,
                    act=rng.choice(["none", "silu", "gelu", "sigmoid", "relu"]), bias=rng.random() < 0.6,
                    residual=op != "linear_grad" and rng.random() < 0.5)
    qk = rng.choice([1, 2, 4, 8, 16])
    heads = qk * rng.choice([h for h in (1, 1, 2, 4) if qk * h <= 16])
    d = rng.choice([(128, 128), (64, 64), (64, 128), (32, 64), (80, 112), (rng.randint(9, 128), rng.randint(9, 128))])
    if op == "delta_step":
        n = _log(rng, 1, 256)
        return dict(op=op, type=t, seqs=n, slots=n + rng.randint(0, 64), heads=heads, qk_heads=qk, dk=d[0], dv=d[1])
    packed = rng.random() < 0.4
    seqs = _log(rng, 1, 64)
    tokens = _log(rng, 256, 16384)
    if not packed:
        tokens = max(1, tokens // seqs) * seqs
    return dict(op=op, type=t, seqs=seqs, tokens=tokens, heads=heads, qk_heads=qk, dk=d[0], dv=d[1], packed=packed,
                state=rng.random() < 0.4)


def prepare(case, seed):
    dev = torch.device("cuda")
    gen = torch.Generator(device=dev).manual_seed(seed)
    dt = TYPES[case["type"]]

    def normal(*shape, scale=1.0, shift=0.0, dtype=dt):
        return (torch.randn(shape, generator=gen, device=dev) * scale + shift).to(dtype)

    s = dict(case=case)
    op = case["op"]
    if op.startswith("rms"):
        rows, n = case["rows"], case["n"]
        x = normal(rows, n, scale=1.5, shift=0.25)
        s.update(weight=normal(n, scale=0.1, shift=1.0), eps=1e-5)
        if op == "rms_grad":        # what the forward pass returned
            s.update(h=x, rstd=(x.float().square().mean(1) + s["eps"]).rsqrt(), dy=normal(rows, n),
                     dh=normal(rows, n) if case["residual"] else None)
        else:
            s.update(x=x, residual=normal(rows, n) if case["residual"] else None)
        return s
    if op.startswith("linear"):
        rows, n_in, n_out = case["rows"], case["n_in"], case["n_out"]
        s.update(x=normal(rows, n_in), weight=normal(n_out, n_in, scale=n_in ** -0.5),
                 bias=normal(n_out, scale=0.3) if case["bias"] else None,
                 residual=normal(rows, n_out) if case["residual"] else None,
                 act=None if case["act"] == "none" else case["act"])
        if op == "linear_grad":
            s["dy"] = normal(rows, n_out)
        if op == "linear_8bit":     # as a model holds its weights, and as a norm has left its rows
            s["x"], s["x_scale"] = _rows_8bit(s["x"].float())
            s["weight"], s["weight_scale"] = _rows_8bit(s["weight"].float())
        return s
    B, H, Hk, dk, dv = case["seqs"], case["heads"], case["qk_heads"], case["dk"], case["dv"]
    s["scale"] = dk ** -0.5

    def inputs(lead):
        # keys and queries of length one; decays from a few points to thousands; how much of a value is written
        q, k = (torch.nn.functional.normalize(normal(*lead, Hk, dk, shift=0.2, dtype=torch.float32), dim=-1) for _ in range(2))
        half = torch.rand((*lead, H), generator=gen, device=dev) * 7.0 + 1.0 * torch.arange(H, device=dev) / H
        s.update(q=(q * dk ** 0.5).to(dt), k=k.to(dt), v=normal(*lead, H, dv), g=(-torch.exp2(-1.0 - half)).to(dt),
                 beta=torch.sigmoid(normal(*lead, H, dtype=torch.float32)).to(dt))

    if op == "delta_step":
        inputs((B,))
        s.update(state=normal(case["slots"], H, dk, dv, dtype=torch.float32),
                 slots=torch.randperm(case["slots"], generator=gen, device=dev)[:B].contiguous())
        return s
    n = case["tokens"]
    if case["packed"]:      # sequences end at random places: some are short, some may be empty
        cuts = torch.randint(0, n + 1, (B - 1,), generator=gen, device=dev).sort().values
        ends = torch.tensor([0, n], device=dev)
        s["offsets"] = torch.cat([ends[:1], cuts, ends[1:]]).long()
        s["longest"] = int((s["offsets"][1:] - s["offsets"][:-1]).max())
        lead = (n,)
    else:
        s["offsets"], s["longest"] = None, n // B
        lead = (B, n // B)
    inputs(lead)
    s["s0"] = normal(B, H, dk, dv, dtype=torch.float32) if case["state"] else None
    if op == "delta_grad":
        s["do"] = normal(*lead, H, dv)
        s["ds"] = normal(B, H, dk, dv, dtype=torch.float32) if case["state"] else None
    return s


def work(case):
    e, op = SIZE[case["type"]], case["op"]
    if op.startswith("rms"):
        r, n, more = case["rows"], case["n"], case["residual"]
        if op == "rms_grad":
            return dict(bytes=(3 + more) * e * r * n + 2 * e * n + 4 * r, flops=9 * r * n)
        return dict(bytes=((1 + 2 * more) * e + (1 if op == "rms_8bit" else e)) * r * n + e * n + 4 * r, flops=5 * r * n)
    if op.startswith("linear"):
        r, i, o = case["rows"], case["n_in"], case["n_out"]
        if op == "linear_grad":
            formed = case["act"] != "none"
            return dict(bytes=e * (2 * r * i + 2 * i * o + r * o), flops=(6 if formed else 4) * r * i * o)
        held = 1 if op == "linear_8bit" else e
        return dict(bytes=held * (r * i + i * o) + e * r * o * (1 + case["residual"]), flops=2 * r * i * o)
    B, H, Hk, dk, dv = case["seqs"], case["heads"], case["qk_heads"], case["dk"], case["dv"]
    states = 4 * B * H * dk * dv
    token = e * (2 * Hk * dk + H * (dv + 2))      # q, k, v, g and beta
    if op == "delta_step":
        return dict(bytes=2 * states + B * (token + e * H * dv), flops=6 * B * H * dk * dv)
    n = case["tokens"]
    if op == "delta":
        return dict(bytes=n * (token + e * H * dv) + states * (1 + case["state"]), flops=6 * n * H * dk * dv)
    return dict(bytes=n * (2 * token + e * H * dv) + states * 3 * case["state"], flops=18 * n * H * dk * dv)


# ------------------------------------------------------------------ one pass
def run(s):
    return (_run_own if own else _run_plain)(s)


def _run_own(s):
    import paper_2607_03574_amd as nd
    op = s["case"]["op"]
    if op == "rms":
        return nd.rms_norm(s["x"], s["weight"], s["residual"], s["eps"])
    if op == "rms_grad":
        return nd.rms_norm_grad(s["dy"], s["h"], s["weight"], s["rstd"], s["dh"])
    if op == "rms_8bit":
        y, scale, h = nd.rms_norm_8bit(s["x"], s["weight"], s["residual"], s["eps"])
        return _held(y, scale, s), scale, h
    if op == "linear":
        return nd.linear(s["x"], s["weight"], s["bias"], s["act"], s["residual"])
    if op == "linear_grad":
        return nd.linear_grad(s["dy"], s["x"], s["weight"], s["bias"], s["act"])
    if op == "linear_8bit":
        return nd.linear_8bit(s["x"], s["x_scale"], s["weight"], s["weight_scale"], s["bias"], s["act"], s["residual"],
                              dtype=TYPES[s["case"]["type"]])
    if op == "delta_step":
        o = nd.delta_attention_step(s["q"], s["k"], s["v"], s["g"], s["beta"], s["state"], slots=s["slots"],
                                    scale=s["scale"])
        return o, s["state"]
    if op == "delta":
        return nd.delta_attention(s["q"], s["k"], s["v"], s["g"], s["beta"], offsets=s["offsets"], scale=s["scale"],
                                  initial_state=s["s0"], final_state=True)
    return nd.delta_attention_grad(s["do"], s["q"], s["k"], s["v"], s["g"], s["beta"], offsets=s["offsets"],
                                   scale=s["scale"], initial_state=s["s0"], grad_final_state=s["ds"])


def _run_plain(s):
    op = s["case"]["op"]
    dt = TYPES[s["case"]["type"]]
    if op == "rms_grad":
        dy = s["dy"].float()
        hh = s["h"].float() * s["rstd"][:, None]
        g = dy * s["weight"].float()
        dx = (g - hh * (g * hh).mean(1, keepdim=True)) * s["rstd"][:, None]
        if s["dh"] is not None:
            dx = dx + s["dh"].float()
        return dx.to(dt), (dy * hh).sum(0).to(dt)
    if op.startswith("rms"):
        h = s["x"] if s["residual"] is None else (s["x"].float() + s["residual"].float()).to(dt)
        rstd = (h.float().square().mean(1) + s["eps"]).rsqrt()
        y = h.float() * rstd[:, None] * s["weight"].float()
        if op == "rms":
            return y.to(dt), h, rstd
        y, scale = _rows_8bit(y)
        return _held(y, scale, s), scale, h
    if op.startswith("linear"):
        x, w = s["x"].float(), s["weight"].float()
        if op == "linear_8bit":
            x, w = x * s["x_scale"][:, None], w * s["weight_scale"][:, None]
        z = None
        if op != "linear_grad" or s["act"] is not None:
            z = x @ w.T
            if s["bias"] is not None:
                z = z + s["bias"].float()
        if op != "linear_grad":
            y = _act(z, s["act"])[0]
            return (y if s["residual"] is None else y + s["residual"].float()).to(dt)
        dz = s["dy"].float()
        if s["act"] is not None:
            dz = dz * _act(z, s["act"])[1]
        return (dz @ w).to(dt), (dz.T @ x).to(dt), None if s["bias"] is None else dz.sum(0).to(dt)
    group = s["case"]["heads"] // s["case"]["qk_heads"]
    if op == "delta_step":
        q, k = (s[n].float().repeat_interleave(group, dim=1) for n in ("q", "k"))
        S = s["state"][s["slots"]] * torch.exp(s["g"].float())[..., None, None]
        u = (s["v"].float() - torch.matmul(k[..., None, :], S)[..., 0, :]) * s["beta"].float()[..., None]
        S = S + k[..., :, None] * u[..., None, :]
        s["state"][s["slots"]] = S
        return (torch.matmul(q[..., None, :], S)[..., 0, :] * s["scale"]).to(dt), s["state"]
    if op == "delta":
        o, S = _delta(s, *(s[n] for n in ("q", "k", "v", "g", "beta")), s["s0"])
        return o.to(dt), S
    names = ("q", "k", "v", "g", "beta")
    with torch.enable_grad():
        leaves = [s[n].float().requires_grad_() for n in names]
        if s["s0"] is not None:
            leaves.append(s["s0"].detach().requires_grad_())
        o, S = _delta(s, *leaves[:5], leaves[5] if len(leaves) > 5 else None)
        outs, into = ((o, S), (s["do"].float(), s["ds"])) if s["ds"] is not None else ((o,), (s["do"].float(),))
        found = torch.autograd.grad(outs, leaves, into)
    return tuple(x.to(dt) for x in found[:5]) + (found[5] if len(found) > 5 else None,)


def _rows_8bit(y):
    """Rows in e4m3 (whose largest value is 448) and their scales."""
    scale = y.abs().amax(1).clamp(min=448.0 * 2.0 ** -126) / 448.0
    return (y / scale[:, None]).to(E4M3), scale


def _held(y, scale, s):
    """The values that 8-bit rows stand for."""
    return (y.float() * scale[:, None]).to(TYPES[s["case"]["type"]])


def _act(z, act):
    """An activation's value and slope."""
    if act is None:
        return z, torch.ones_like(z)
    if act == "relu":
        return z.clamp(min=0), (z > 0).float()
    if act == "gelu":
        p = 0.5 * (1.0 + torch.erf(z * math.sqrt(0.5)))
        return z * p, p + z * torch.exp(-0.5 * z * z) * (2.0 * math.pi) ** -0.5
    p = torch.sigmoid(z)
    if act == "sigmoid":
        return p, p * (1.0 - p)
    return z * p, p * (1.0 + z * (1.0 - p))


def _places(s):
    """Sequences in rows of one length (a multiple of CHUNK), moved to their ends: for each place its token, and whether
    it has one."""
    dev, B = s["q"].device, s["case"]["seqs"]
    T = -(-s["longest"] // CHUNK) * CHUNK
    t = torch.arange(T, device=dev)[None]
    if s["offsets"] is None:
        first, length = torch.arange(B, device=dev) * s["longest"], torch.full((B,), s["longest"], device=dev)
    else:
        first, length = s["offsets"][:-1], s["offsets"][1:] - s["offsets"][:-1]
    pos = t - (T - length)[:, None]
    return (first[:, None] + pos.clamp(min=0)).clamp(max=max(s["case"]["tokens"] - 1, 0)), pos >= 0


def _delta(s, q, k, v, g, beta, s0):
    """(o, final state) in 32 bits.  In a block of CHUNK tokens, with G the running sum of g, L_ij = exp(G_i - G_j) and
    A_ij = beta_i L_ij k_i.k_j for j < i: what the tokens write is U = (I + A)^-1 diag(beta) (V - exp(G) K S), and the
    block turns the state S into exp(G_last) S + sum_j exp(G_last - G_j) k_j^T u_j.  A token that a row lacks writes
    nothing."""
    at, there = _places(s)
    c, group = s["case"], s["case"]["heads"] // s["case"]["qk_heads"]

    def blocks(x, shared, d):
        x = x.float().reshape(c["tokens"], -1, d)
        x = torch.where(there[..., None, None], x[at], 0.0)
        x = x.repeat_interleave(group, dim=2) if shared else x
        return x.transpose(1, 2).unflatten(2, (-1, CHUNK))        # [B, H, N, CHUNK, d]

    q, k = (blocks(x, True, c["dk"]) for x in (q, k))
    v, g, beta = blocks(v, False, c["dv"]), blocks(g, False, 1), blocks(beta, False, 1)
    G = g.double().cumsum(3)
    low = torch.ones(CHUNK, CHUNK, device=q.device, dtype=torch.bool).tril()
    far = torch.where(low, G - G.transpose(3, 4), 0.0)
    L = torch.where(low, torch.exp(far), 0.0).float()
    rise, fall, whole = torch.exp(G).float(), torch.exp(G[..., -1:, :] - G).float(), torch.exp(G[..., -1:, :]).float()
    A = beta * L * torch.matmul(k, k.transpose(3, 4))
    T = _inverse(torch.where(low.tril(-1), A, 0.0).double()).float()
    W, U = torch.matmul(T, beta * rise * k), torch.matmul(T, beta * v)
    kt = (k * fall).transpose(3, 4)
    keep = whole * torch.eye(c["dk"], device=q.device) - torch.matmul(kt, W)
    add = torch.matmul(kt, U)
    S = s0 if s0 is not None else torch.zeros(*q.shape[:2], c["dk"], c["dv"], device=q.device)
    enters = []
    for n in range(q.shape[2]):
        enters.append(S)
        S = torch.matmul(keep[:, :, n], S) + add[:, :, n]
    if not enters:
        return torch.zeros_like(v).reshape(*s["v"].shape), S
    S0 = torch.stack(enters, 2)
    U = U - torch.matmul(W, S0)
    o = torch.matmul(q * rise, S0) + torch.matmul(torch.matmul(q, k.transpose(3, 4)) * L, U)
    o = (o * s["scale"]).flatten(2, 3).transpose(1, 2)
    return o[there].reshape(s["v"].shape), S


def _inverse(A):
    """(I + A)^-1 of strictly lower triangular matrices: the product of I + A^(2^i), with -A."""
    eye = torch.eye(CHUNK, device=A.device, dtype=A.dtype)
    power, T = -A, eye - A
    for _ in range(CHUNK.bit_length() - 2):
        power = torch.matmul(power, power)
        T = T + torch.matmul(T, power)
    return T


# ------------------------------------------------------------------ in 64 bits, from the definitions
def exact(case, seed):
    s = prepare(case, seed)
    d = {n: x.double() if isinstance(x, torch.Tensor) and x.is_floating_point() else x for n, x in s.items()}
    op, dt = case["op"], TYPES[case["type"]]
    if op == "rms_grad":
        # the gradient through y = h rstd w, rstd as it was given, and what comes along h itself
        n = case["n"]
        g = d["dy"] * d["weight"]
        along = torch.einsum("rn,rn->r", g, d["h"])[:, None] / n
        dx = d["rstd"][:, None] * g - d["rstd"][:, None] ** 3 * d["h"] * along
        return (dx if s["dh"] is None else dx + d["dh"]), torch.einsum("rn,rn,r->n", d["dy"], d["h"], d["rstd"])
    if op.startswith("rms"):
        h = d["x"] if s["residual"] is None else (d["x"] + d["residual"]).to(dt).double()
        rstd = 1.0 / torch.sqrt(torch.linalg.vector_norm(h, dim=1) ** 2 / case["n"] + d["eps"])
        y = torch.einsum("rn,r,n->rn", h, rstd, d["weight"])
        if op == "rms":
            return y, h, rstd
        scale = torch.linalg.vector_norm(y, float("inf"), dim=1).clamp(min=448 * 2.0 ** -126) / 448
        q = torch.einsum("rn,r->rn", y, 1.0 / scale)
        step = torch.exp2(torch.floor(torch.log2(q.abs().clamp(min=2.0 ** -6))) - 3)     # of e4m3 around a value
        return torch.round(q / step) * step * scale[:, None], scale, h
    if op.startswith("linear"):
        if op == "linear_8bit":
            d["x"], d["weight"] = s["x"].double(), s["weight"].double()
            z = torch.nn.functional.linear(d["x"], d["weight"]) * torch.outer(d["x_scale"], d["weight_scale"])
            z = z if s["bias"] is None else z + d["bias"]
        else:
            z = torch.nn.functional.linear(d["x"], d["weight"], d["bias"])
        act = {None: lambda t: t, "relu": torch.relu, "gelu": torch.nn.functional.gelu, "sigmoid": lambda t: 1 / (1 + torch.exp(-t)),
               "silu": lambda t: t / (1 + torch.exp(-t))}[s["act"]]
        if op != "linear_grad":
            return act(z) if s["residual"] is None else act(z) + d["residual"]
        with torch.enable_grad():
            z = z.detach().requires_grad_()
            (dz,) = torch.autograd.grad(act(z), z, d["dy"])
        return dz.mm(d["weight"]), dz.T.mm(d["x"]), None if s["bias"] is None else dz.sum(0)
    H, group = case["heads"], case["heads"] // case["qk_heads"]
    wide = torch.arange(H, device="cuda") // group       # a head's queries and keys
    if op == "delta_step":
        S = d["state"][d["slots"]] * torch.exp(d["g"])[..., None, None]
        k = d["k"][:, wide]
        miss = d["v"] - torch.einsum("bhi,bhij->bhj", k, S)
        S = S + torch.einsum("bhi,bhj,bh->bhij", k, miss, d["beta"])
        d["state"][d["slots"]] = S
        return torch.einsum("bhi,bhij->bhj", d["q"][:, wide], S) * s["scale"], d["state"]
    # token by token; sequences of one length together
    n, B, dk, dv = case["tokens"], case["seqs"], case["dk"], case["dv"]
    if case["packed"]:
        bounds = s["offsets"].tolist()
        parts = [(torch.arange(bounds[i], bounds[i + 1], device="cuda")[None], [i]) for i in range(B)]
    else:
        parts = [(torch.arange(n, device="cuda").view(B, n // B), list(range(B)))]
    flat = {x: d[x].reshape(n, *d[x].shape[len(s["q"].shape) - 2:]) for x in ("q", "k", "v", "g", "beta")}
    gradient = op == "delta_grad"
    do = d["do"].reshape(n, H, dv) * s["scale"] if gradient else None
    o = torch.zeros(n, H, dv, dtype=torch.float64, device="cuda")
    out = {x: torch.zeros(n, H, w, dtype=torch.float64, device="cuda") for x, w in (("q", dk), ("k", dk), ("v", dv), ("g", 1), ("beta", 1))}
    S1 = torch.zeros(B, H, dk, dv, dtype=torch.float64, device="cuda")
    if s["s0"] is not None:
        S1 += d["s0"]
    dS0 = torch.zeros_like(S1)
    for at, which in parts:
        T = at.shape[1]
        q, k = flat["q"][at][:, :, wide].unsqueeze(-2), flat["k"][at][:, :, wide].unsqueeze(-2)      # [b, T, H, 1, dk]
        v, beta, a = flat["v"][at].unsqueeze(-2), flat["beta"][at][..., None, None], torch.exp(flat["g"][at])[..., None, None]
        S = S1[which]
        decayed = torch.empty((T if gradient else 0, *S.shape), dtype=torch.float64, device="cuda")
        u = torch.empty_like(v) if gradient else None
        for t in range(T):
            S = S * a[:, t]
            w = (v[:, t] - k[:, t] @ S) * beta[:, t]
            if gradient:
                decayed[t], u[:, t] = S, w
            S = S + k[:, t].transpose(-1, -2) * w
            if not gradient:
                o[at[:, t]] = (q[:, t] @ S)[..., 0, :] * s["scale"]
        S1[which] = S
        if not gradient:
            continue
        dS = d["ds"][which] if s["ds"] is not None else torch.zeros_like(S)
        dO = do[at].unsqueeze(-2)
        for t in reversed(range(T)):
            kt, Sd = k[:, t].transpose(-1, -2), decayed[t]
            out["q"][at[:, t]] = (dO[:, t] @ (Sd + kt * u[:, t]).transpose(-1, -2))[..., 0, :]
            dS = dS + q[:, t].transpose(-1, -2) * dO[:, t]
            du = k[:, t] @ dS                           # of what the token wrote
            dw = du * beta[:, t]                        # of v - k S
            out["v"][at[:, t]] = dw[..., 0, :]
            out["beta"][at[:, t]] = (du * (v[:, t] - k[:, t] @ Sd)).sum(-1)
            out["k"][at[:, t]] = (u[:, t] @ dS.transpose(-1, -2) - dw @ Sd.transpose(-1, -2))[..., 0, :]
            dS = dS - kt * dw
            out["g"][at[:, t]] = (dS * Sd).sum((-1, -2))[..., None]
            dS = dS * a[:, t]
        dS0[which] = dS
    if not gradient:
        return o.reshape(s["v"].shape), S1
    for x in ("q", "k"):
        out[x] = out[x].unflatten(1, (H // group, group)).sum(2)
    return tuple(out[x].reshape(s[x].shape) for x in ("q", "k", "v", "g", "beta")) + (dS0 if s["s0"] is not None else None,)

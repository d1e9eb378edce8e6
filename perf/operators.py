"""The operators of a sequence encoder whose output feeds the replay's parameters, as timed cases:
layer norm, linear attention with a decay for each head, and the gated feed-forward projections.

`run` computes them in plain torch operations in 32 bits, or, with `own` set, through this package's
entry points.  Sizes run from one token of a stream to training batches and long observation series.
"""
import math

import torch

own = False

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SIZE = {"f32": 4, "bf16": 2, "f16": 2}
CHUNK = 64      # tokens per block of the plain chunked attention


# ------------------------------------------------------------------ cases
def listed():
    return [
        # one token of four streams: what a norm costs between two steps of a stream
        dict(name="norm_token", op="norm", type="bf16", rows=4, n=1024),
        # the norm in front of a block, 16 series of 2048 points at once
        dict(name="norm_batch", op="norm", type="bf16", rows=32768, n=2048),
        # its gradient in a training step
        dict(name="norm_grad_batch", op="norm_grad", type="bf16", rows=16384, n=2048),
        # a small model in single precision, odd sizes
        dict(name="norm_grad_odd", op="norm_grad", type="f32", rows=5003, n=1000),
        # one long series read at once, the state kept for the stream that follows
        dict(name="attention_long", op="attention", type="bf16", seqs=1, tokens=16384, heads=16, kv_heads=16, dk=128,
             dv=128, packed=False, state=False),
        # 37 series of different lengths in one pass, four query heads sharing a key
        dict(name="attention_packed", op="attention", type="bf16", seqs=37, tokens=9001, heads=16, kv_heads=4, dk=64,
             dv=128, packed=True, state=False),
        # the gradient in a training step
        dict(name="attention_grad_batch", op="attention_grad", type="bf16", seqs=8, tokens=16384, heads=16, kv_heads=16,
             dk=128, dv=128, packed=False, state=False),
        # a small model in single precision, series cut in pieces: states go in and their gradients come out
        dict(name="attention_grad_odd", op="attention_grad", type="f32", seqs=3, tokens=2331, heads=6, kv_heads=2, dk=40,
             dv=72, packed=False, state=True),
        # one new point of 192 streams that live in 256 slots
        dict(name="attention_step", op="step", type="bf16", seqs=192, slots=256, heads=16, kv_heads=16, dk=128, dv=128),
        # the feed-forward of one point of 17 streams: weights are what is read
        dict(name="ffn_few", op="ffn", type="bf16", rows=17, n_in=1024, n_out=4096),
        # the feed-forward of a batch
        dict(name="ffn_batch", op="ffn", type="bf16", rows=8192, n_in=2048, n_out=8192),
        # its gradient in a training step
        dict(name="ffn_grad_batch", op="ffn_grad", type="bf16", rows=4096, n_in=1024, n_out=4096),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["norm", "norm_grad", "attention", "attention", "attention_grad", "step", "ffn", "ffn_grad"])
    t = rng.choice(["bf16", "bf16", "bf16", "f16", "f32"])
    if op in ("norm", "norm_grad"):
        n = _log(rng, 17, 8192)
        return dict(op=op, type=t, rows=_log(rng, 1, min(65536, (1 << 26) // n)), n=n)
    if op in ("ffn", "ffn_grad"):
        n_in, n_out = _log(rng, 48, 2048), _log(rng, 48, 8192)
        if rng.random() < 0.5:      # widths of most models are multiples of 64
            n_in, n_out = max(64, n_in // 64 * 64), max(64, n_out // 64 * 64)
        return dict(op=op, type=t, rows=_log(rng, 1, 8192 if op == "ffn" else 4096), n_in=n_in, n_out=n_out)
    kv = rng.choice([1, 2, 4, 8, 16])
    heads = kv * rng.choice([h for h in (1, 1, 2, 4) if kv * h <= 16])
    d = rng.choice([(128, 128), (64, 64), (64, 128), (32, 64), (80, 112), (rng.randint(9, 128), rng.randint(9, 128))])
    if op == "step":
        n = _log(rng, 1, 256)
        return dict(op=op, type=t, seqs=n, slots=n + rng.randint(0, 64), heads=heads, kv_heads=kv, dk=d[0], dv=d[1])
    packed = rng.random() < 0.4
    seqs = _log(rng, 1, 64)
    tokens = _log(rng, 256, 16384)
    if not packed:
        tokens = max(1, tokens // seqs) * seqs
    return dict(op=op, type=t, seqs=seqs, tokens=tokens, heads=heads, kv_heads=kv, dk=d[0], dv=d[1], packed=packed,
                state=rng.random() < 0.4)


def prepare(case, seed):
    dev = torch.device("cuda")
    gen = torch.Generator(device=dev).manual_seed(seed)
    dt = TYPES[case["type"]]

    def normal(*shape, scale=1.0, shift=0.0, dtype=dt):
        return (torch.randn(shape, generator=gen, device=dev) * scale + shift).to(dtype)

    s = dict(case=case)
    op = case["op"]
    if op in ("norm", "norm_grad"):
        rows, n = case["rows"], case["n"]
        s.update(x=normal(rows, n, scale=1.5, shift=0.25), weight=normal(n, scale=0.1, shift=1.0),
                 bias=normal(n, scale=0.1), eps=1e-5)
        if op == "norm_grad":       # the statistics that the forward pass returned
            xf = s["x"].float()
            s["mean"] = xf.mean(1)
            s["rstd"] = (xf.var(1, unbiased=False) + s["eps"]).rsqrt()
            s["dy"] = normal(rows, n)
        return s
    if op in ("ffn", "ffn_grad"):
        rows, n_in, n_out = case["rows"], case["n_in"], case["n_out"]
        s.update(x=normal(rows, n_in), w_gate=normal(n_out, n_in, scale=n_in ** -0.5),
                 w_up=normal(n_out, n_in, scale=n_in ** -0.5))
        if op == "ffn_grad":
            s["dh"] = normal(rows, n_out)
        return s
    B, H, Hk, dk, dv = case["seqs"], case["heads"], case["kv_heads"], case["dk"], case["dv"]
    # half-lives from a few points to thousands, one for each head
    s["log_decay"] = torch.log1p(-torch.exp2(-(4.0 + 7.0 * torch.arange(H, device=dev) / H))).float()
    s["scale"] = dk ** -0.5
    if op == "step":
        s.update(q=normal(B, H, dk), k=normal(B, Hk, dk), v=normal(B, Hk, dv),
                 state=normal(case["slots"], H, dk, dv, dtype=torch.float32),
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
    s.update(q=normal(*lead, H, dk), k=normal(*lead, Hk, dk), v=normal(*lead, Hk, dv))
    s["s0"] = normal(B, H, dk, dv, dtype=torch.float32) if case["state"] else None
    if op == "attention_grad":
        s["do"] = normal(*lead, H, dv)
        s["ds"] = normal(B, H, dk, dv, dtype=torch.float32) if case["state"] else None
    return s


def work(case):
    e, op = SIZE[case["type"]], case["op"]
    if op in ("norm", "norm_grad"):
        r, n = case["rows"], case["n"]
        if op == "norm":
            return dict(bytes=2 * e * r * n + 2 * e * n + 8 * r, flops=8 * r * n)
        return dict(bytes=3 * e * r * n + 3 * e * n + 8 * r, flops=13 * r * n)
    if op in ("ffn", "ffn_grad"):
        r, i, o = case["rows"], case["n_in"], case["n_out"]
        if op == "ffn":
            return dict(bytes=e * (r * i + 2 * i * o + r * o), flops=4 * r * i * o)
        return dict(bytes=e * (2 * r * i + 4 * i * o + r * o), flops=12 * r * i * o)
    B, H, Hk, dk, dv = case["seqs"], case["heads"], case["kv_heads"], case["dk"], case["dv"]
    states = 4 * B * H * dk * dv
    if op == "step":
        return dict(bytes=2 * states + e * B * (H * (dk + dv) + Hk * (dk + dv)), flops=4 * B * H * dk * dv)
    n = case["tokens"]
    if op == "attention":
        return dict(bytes=e * n * (H * (dk + dv) + Hk * (dk + dv)) + states * (1 + case["state"]),
                    flops=4 * n * H * dk * dv)
    return dict(bytes=e * n * (H * (2 * dk + dv) + 2 * Hk * (dk + dv)) + states * 3 * case["state"],
                flops=10 * n * H * dk * dv)


# ------------------------------------------------------------------ one pass
def run(s):
    return (_run_own if own else _run_plain)(s)


def _run_own(s):
    import paper_2607_03574_amd as nd
    op = s["case"]["op"]
    if op == "norm":
        return nd.layer_norm(s["x"], s["weight"], s["bias"], s["eps"])
    if op == "norm_grad":
        return nd.layer_norm_grad(s["dy"], s["x"], s["weight"], s["mean"], s["rstd"])
    if op == "ffn":
        return nd.gated_ffn(s["x"], s["w_gate"], s["w_up"], "silu")
    if op == "ffn_grad":
        return nd.gated_ffn_grad(s["dh"], s["x"], s["w_gate"], s["w_up"], "silu")
    if op == "step":
        o = nd.linear_attention_step(s["q"], s["k"], s["v"], s["log_decay"], s["state"], slots=s["slots"],
                                     scale=s["scale"])
        return o, s["state"]
    if op == "attention":
        return nd.linear_attention(s["q"], s["k"], s["v"], s["log_decay"], offsets=s["offsets"], scale=s["scale"],
                                   initial_state=s["s0"], final_state=True)
    return nd.linear_attention_grad(s["do"], s["q"], s["k"], s["v"], s["log_decay"], offsets=s["offsets"],
                                    scale=s["scale"], initial_state=s["s0"], grad_final_state=s["ds"])


def _run_plain(s):
    op = s["case"]["op"]
    dt = TYPES[s["case"]["type"]]
    if op == "norm":
        x = s["x"].float()
        mean = x.mean(1)
        c = x - mean[:, None]
        rstd = (c.square().mean(1) + s["eps"]).rsqrt()
        return (c * rstd[:, None] * s["weight"].float() + s["bias"].float()).to(dt), mean, rstd
    if op == "norm_grad":
        dy = s["dy"].float()
        xh = (s["x"].float() - s["mean"][:, None]) * s["rstd"][:, None]
        g = dy * s["weight"].float()
        dx = (g - g.mean(1, keepdim=True) - xh * (g * xh).mean(1, keepdim=True)) * s["rstd"][:, None]
        return dx.to(dt), (dy * xh).sum(0).to(dt), dy.sum(0).to(dt)
    if op in ("ffn", "ffn_grad"):
        x, wg, wu = s["x"].float(), s["w_gate"].float(), s["w_up"].float()
        g, u = x @ wg.T, x @ wu.T
        sg = torch.sigmoid(g)
        if op == "ffn":
            return (g * sg * u).to(dt)
        dh = s["dh"].float()
        dg = dh * u * (sg * (1.0 + g * (1.0 - sg)))
        du = dh * (g * sg)
        return (dg @ wg + du @ wu).to(dt), (dg.T @ x).to(dt), (du.T @ x).to(dt)
    H, group = s["case"]["heads"], s["case"]["heads"] // s["case"]["kv_heads"]
    g = s["log_decay"]
    if op == "step":
        q, k, v = s["q"].float(), _shared(s["k"].float(), group), _shared(s["v"].float(), group)
        S = s["state"][s["slots"]] * torch.exp(g)[:, None, None] + k[..., :, None] * v[..., None, :]
        s["state"][s["slots"]] = S
        return (torch.matmul(q[..., None, :], S)[..., 0, :] * s["scale"]).to(dt), s["state"]
    at, there, pos, left, length = _places(s)
    q, k, v = (_padded(s[n].float(), at, there, w) for n, w in (("q", 1), ("k", group), ("v", group)))   # [B, H, T, d]
    rise = _power(g[None, :, None], pos[:, None] + 1.0)[..., None]       # decay from before the sequence to a token
    fall = _power(g[None, :, None], left[:, None])[..., None]            # decay from a token to the sequence's end
    whole = _power(g[None, :], length[:, None])[..., None, None]
    if op == "attention":
        o = _attend(q, k, v, g)
        S = torch.matmul((k * fall).transpose(2, 3), v)
        if s["s0"] is not None:
            o = o + torch.matmul(q, s["s0"]) * rise
            S = S + whole * s["s0"]
        return _unpadded(o * s["scale"], s["q"], at, there).to(dt), S
    do = _padded(s["do"].float(), at, there, 1) * s["scale"]
    dq = _attend(do, v, k, g)
    dk = _attend(v.flip(2), do.flip(2), q.flip(2), g).flip(2)
    dv = _attend(k.flip(2), q.flip(2), do.flip(2), g).flip(2)
    ds0 = None
    if s["s0"] is not None:
        dq = dq + torch.matmul(do, s["s0"].transpose(2, 3)) * rise
        dk = dk + torch.matmul(v, s["ds"].transpose(2, 3)) * fall
        dv = dv + torch.matmul(k, s["ds"]) * fall
        ds0 = torch.matmul((q * rise).transpose(2, 3), do) + whole * s["ds"]
    dk, dv = (x.unflatten(1, (H // group, group)).sum(2) for x in (dk, dv))
    return tuple(_unpadded(x, s["q"], at, there).to(dt) for x in (dq, dk, dv)) + (ds0,)


def _shared(x, group):
    """Heads that several query heads share, once for each of them (last axis but one)."""
    return x.repeat_interleave(group, dim=-2)


def _power(g, n):
    return torch.exp(g * n)


def _places(s):
    """Sequences in rows of one length, moved to their ends: for each place its token, whether it has one, its
    place in its sequence, how many tokens follow it, and each sequence's length."""
    dev, T, B = s["q"].device, s["longest"], s["case"]["seqs"]
    t = torch.arange(T, device=dev)[None]
    if s["offsets"] is None:
        first, length = torch.arange(B, device=dev) * T, torch.full((B,), T, device=dev)
    else:
        first, length = s["offsets"][:-1], s["offsets"][1:] - s["offsets"][:-1]
    pos = t - (T - length)[:, None]
    there = pos >= 0
    return (first[:, None] + pos.clamp(min=0)).clamp(max=s["case"]["tokens"] - 1), there, pos.clamp(min=0).float(), (T - 1 - t).float().expand(B, T), length.float()


def _padded(x, at, there, group):
    x = x.reshape(-1, *x.shape[-2:])
    x = torch.where(there[..., None, None], x[at], 0.0)
    return _shared(x, group).transpose(1, 2).contiguous()


def _unpadded(x, like, at, there):
    x = x.transpose(1, 2)
    return x[there].reshape(*like.shape[:-2], *x.shape[2:])


def _attend(a, b, c, g):
    """out_i = sum over j <= i of exp(g (i - j)) (a_i . b_j) c_j for a, b, c [B, H, T, d], by blocks of CHUNK tokens:
    inside a block by a masked product, across blocks by the sums that each block adds."""
    B, H, T, _ = a.shape
    N = -(-T // CHUNK)
    a, b, c = (torch.nn.functional.pad(x, (0, 0, 0, N * CHUNK - T)).unflatten(2, (N, CHUNK)) for x in (a, b, c))
    i = torch.arange(CHUNK, device=a.device, dtype=torch.float32)
    far = i[:, None] - i[None]
    inside = torch.where(far >= 0, _power(g[:, None, None], far.clamp(min=0)), 0.0)[:, None]
    out = torch.matmul(torch.matmul(a, b.transpose(3, 4)) * inside, c)
    sums = torch.matmul((b * _power(g[:, None], CHUNK - 1 - i)[:, None, :, None]).transpose(3, 4), c)   # [B, H, N, d, d]
    n = torch.arange(N, device=a.device, dtype=torch.float32)
    gap = n[:, None] - n[None] - 1
    across = torch.where(gap >= 0, _power(g[:, None, None], CHUNK * gap.clamp(min=0)), 0.0)
    before = torch.matmul(across, sums.flatten(3)).view(sums.shape)
    out = out + torch.matmul(a, before) * _power(g[:, None], i + 1)[:, None, :, None]
    return out.flatten(2, 3)[:, :, :T]


# ------------------------------------------------------------------ in 64 bits, from the definitions
def exact(case, seed):
    s = prepare(case, seed)
    d = {k: v.double() if isinstance(v, torch.Tensor) and v.is_floating_point() else v for k, v in s.items()}
    op = case["op"]
    if op == "norm":
        var, mean = torch.var_mean(d["x"], dim=1, correction=0)
        rstd = 1.0 / torch.sqrt(var + d["eps"])
        return torch.addcmul(d["bias"], (d["x"] - mean[:, None]) * rstd[:, None], d["weight"]), mean, rstd
    if op == "norm_grad":
        # the gradient through y = (x - mean) rstd w + b, the statistics as they were given
        xh = (d["x"] - d["mean"][:, None]) * d["rstd"][:, None]
        g = d["dy"] * d["weight"]
        n = case["n"]
        along = torch.einsum("rn,rn->r", g, xh)[:, None] / n
        dx = d["rstd"][:, None] * (g - (g.sum(1) / n)[:, None] - xh * along)
        return dx, torch.einsum("rn,rn->n", d["dy"], xh), d["dy"].sum(0)
    if op in ("ffn", "ffn_grad"):
        G = torch.nn.functional.linear(d["x"], d["w_gate"])
        U = torch.nn.functional.linear(d["x"], d["w_up"])
        sig = 1.0 / (1.0 + torch.exp(-G))
        act = G * sig
        if op == "ffn":
            return act * U
        dG = d["dh"] * U * (sig + act * (1.0 - sig))
        dU = d["dh"] * act
        return torch.addmm(dG @ d["w_gate"], dU, d["w_up"]), dG.T.mm(d["x"]), dU.T.mm(d["x"])
    H, Hk = case["heads"], case["kv_heads"]
    lam = torch.exp(d["log_decay"])
    if op == "step":
        o = torch.zeros(case["seqs"], H, case["dv"], dtype=torch.float64, device="cuda")
        for h in range(H):
            c = h * Hk // H
            S = lam[h] * d["state"][d["slots"], h] + torch.einsum("bi,bj->bij", d["k"][:, c], d["v"][:, c])
            d["state"][d["slots"], h] = S
            o[:, h] = torch.einsum("bij,bi->bj", S, d["q"][:, h]) * s["scale"]
        return o, d["state"]
    B, n = case["seqs"], case["tokens"]
    bounds = [i * (n // B) for i in range(B + 1)] if s["offsets"] is None else s["offsets"].tolist()
    q, k, v = (d[x].reshape(n, -1, d[x].shape[-1]) for x in ("q", "k", "v"))
    gradient = op == "attention_grad"
    do = d["do"].reshape(n, H, -1) * s["scale"] if gradient else None
    o = torch.zeros(n, H, case["dv"], dtype=torch.float64, device="cuda")
    S1 = torch.zeros(B, H, case["dk"], case["dv"], dtype=torch.float64, device="cuda")
    dq, dk, dv, dS0 = (torch.zeros_like(x) for x in (q, k, v, S1))
    for m in range(B):
        lo, T = bounds[m], bounds[m + 1] - bounds[m]
        t = torch.arange(T, dtype=torch.float64, device="cuda")
        for h in range(H):
            c, gl = h * Hk // H, d["log_decay"][h]
            first, last = torch.exp(gl * (t + 1)), torch.exp(gl * (T - 1 - t))
            Q, K, V = q[lo:lo + T, h], k[lo:lo + T, c], v[lo:lo + T, c]
            if not gradient:
                S1[m, h] = K.T @ (V * last[:, None])
                if s["s0"] is not None:
                    S1[m, h] += torch.exp(gl * T) * d["s0"][m, h]
            for r in range(0, T, 2048):
                e = min(T, r + 2048)        # rows r..e see the tokens before e
                D = torch.tril(torch.exp(gl * (t[r:e, None] - t[None, :e]).clamp(min=0)), diagonal=r)
                if not gradient:
                    o[lo + r:lo + e, h] = ((Q[r:e] @ K[:e].T) * D) @ V[:e] * s["scale"]
                    continue
                dO = do[lo + r:lo + e, h]
                A, dA = (Q[r:e] @ K[:e].T) * D, (dO @ V[:e].T) * D
                dq[lo + r:lo + e, h] = dA @ K[:e]
                dk[lo:lo + e, c] += dA.T @ Q[r:e]
                dv[lo:lo + e, c] += A.T @ dO
            if s["s0"] is not None:
                if not gradient:
                    o[lo:lo + T, h] += (Q @ d["s0"][m, h]) * first[:, None] * s["scale"]
                    continue
                dO = do[lo:lo + T, h]
                dq[lo:lo + T, h] += (dO @ d["s0"][m, h].T) * first[:, None]
                dk[lo:lo + T, c] += (V @ d["ds"][m, h].T) * last[:, None]
                dv[lo:lo + T, c] += (K @ d["ds"][m, h]) * last[:, None]
                dS0[m, h] = (Q * first[:, None]).T @ dO + torch.exp(gl * T) * d["ds"][m, h]
    if not gradient:
        return o.reshape(*s["q"].shape[:-1], -1), S1
    return (dq.reshape(s["q"].shape), dk.reshape(s["k"].shape), dv.reshape(s["v"].shape),
            dS0 if s["s0"] is not None else None)

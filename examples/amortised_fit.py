"""Amortised calibration: an encoder reads noisy logistic growth series and answers
with the program's parameters (r, K, x0, sigma), trained through the replay's
exact gradients; then new points of the same series arrive one by one.

One encoder block: layer norm, linear attention with a decay for each head, gated
feed-forward (torch_api.layer_norm, linear_attention, gated_ffn; the plain
projections are torch's).  The loss of a series is the program's negative
log-likelihood at the encoder's answer (torch_api.replay_loss).  A stream keeps
the attention's state: each new point costs one linear_attention_step.

    python examples/amortised_fit.py [--series 8] [--points 200] [--steps 60]
"""
import argparse
import os
import sys

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2607_03574_amd as nd  # noqa: E402
from paper_2607_03574_amd import torch_api  # noqa: E402
from workloads import configs  # noqa: E402

CENTRE = torch.tensor([2.0, 10.0, 0.5, 0.3], dtype=torch.float64)      # the answer before training


class Encoder(torch.nn.Module):
    def __init__(self, width=64, heads=4, kv_heads=2, d=32, hidden=160):
        super().__init__()
        self.shape = (heads, kv_heads, d)
        linear = torch.nn.Linear
        self.read, self.answer = linear(2, width), linear(width, 4)
        self.qkv, self.mix = linear(width, (heads + 2 * kv_heads) * d, bias=False), linear(heads * d, width, bias=False)
        self.gate, self.up, self.down = (linear(width, hidden, bias=False), linear(width, hidden, bias=False),
                                         linear(hidden, width, bias=False))
        self.norms = torch.nn.ParameterList([torch.nn.Parameter(torch.ones(width)) for _ in range(3)])
        self.register_buffer("log_decay", torch.log1p(-torch.exp2(-3.0 - 2.0 * torch.arange(heads))))
        torch.nn.init.zeros_(self.answer.weight)
        torch.nn.init.zeros_(self.answer.bias)

    def heads(self, x):
        """Queries, keys and values of x [.., width]: views of one product."""
        H, Hk, d = self.shape
        qkv = self.qkv(torch_api.layer_norm(x, self.norms[0]))
        return [t.unflatten(-1, (-1, d)) for t in qkv.split([H * d, Hk * d, Hk * d], dim=-1)]

    def rest(self, x, attended):
        x = x + self.mix(attended.flatten(-2))
        y = torch_api.layer_norm(x, self.norms[1])
        x = x + self.down(torch_api.gated_ffn(y, self.gate.weight, self.up.weight))
        theta = self.answer(torch_api.layer_norm(x, self.norms[2]))
        return CENTRE.to(x.device) * torch.exp(theta.double())

    def forward(self, points):
        """points [series, T, 2] -> the answer after every point [series, T, 4], and the state."""
        x = self.read(points)
        o, state = torch_api.linear_attention(*self.heads(x), self.log_decay)
        return self.rest(x, o), state

    @torch.no_grad()
    def step(self, point, state):
        """One new point [series, 2]; updates the state in place."""
        x = self.read(point)
        q, k, v = (t.contiguous() for t in self.heads(x))
        return self.rest(x, nd.linear_attention_step(q, k, v, self.log_decay, state))


def series(n, T, seed=0):
    """n noisy paths with parameters around CENTRE, as the encoder reads them (value / 10, time)."""
    rng = np.random.default_rng(seed)
    theta = CENTRE.numpy() * 2.0 ** rng.uniform(-1, 1, size=(n, 4))
    y = np.stack([configs.logistic_truth_path(t, T) + rng.normal(0.0, t[3], T) for t in theta])
    return theta, y


def points_of(y):
    t = torch.arange(y.shape[1], device=y.device) / y.shape[1]
    return torch.stack([y.float() / 10.0, t.expand(y.shape[0], -1)], -1).contiguous()


def main(n=8, T=200, steps=60, lr=3e-3, seed=0, report=print):
    """Trains; returns the mean loss before each step, and how far the streamed answers are from those of the whole
    series read at once (relative)."""
    torch.manual_seed(seed)
    _, y = series(n, T, seed)
    obs = torch.tensor(y, device="cuda")
    points = points_of(obs)
    tape = nd.tape_upload(nd.tape_build(configs.logistic_program(T)))
    workspace = torch.empty(max(nd.workspace_bytes(tape, 1), 8), dtype=torch.uint8, device="cuda")
    model = Encoder().cuda()
    optimiser = torch.optim.Adam(model.parameters(), lr=lr)
    history = []
    for i in range(steps):
        answers, _ = model(points)
        theta = answers[:, -1].contiguous()         # after the last point
        loss = torch.stack([torch_api.replay_loss(tape, theta[s:s + 1], obs[s], workspace).mean() for s in range(n)]).mean() / T
        optimiser.zero_grad()
        loss.backward()
        optimiser.step()
        history.append(float(loss.detach()))
        if i % 10 == 0:
            report(f"step {i:4d}  loss per point {history[-1]:.4f}", flush=True)
    # the first half at once, the rest point by point
    with torch.no_grad():
        whole, _ = model(points)
        _, state = model(points[:, :T // 2].contiguous())
    streamed = torch.stack([model.step(points[:, t], state) for t in range(T // 2, T)], 1)
    want = whole[:, T // 2:]
    apart = float(((streamed - want).norm() / want.norm()))
    report(f"loss per point {history[0]:.4f} -> {history[-1]:.4f}; streamed answers within {apart:.1e}", flush=True)
    return history, apart


if __name__ == "__main__":
    ap = argparse.ArgumentParser()
    ap.add_argument("--series", type=int, default=8)
    ap.add_argument("--points", type=int, default=200)
    ap.add_argument("--steps", type=int, default=60)
    a = ap.parse_args()
    main(a.series, a.points, a.steps)

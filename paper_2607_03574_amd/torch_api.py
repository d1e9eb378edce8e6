"""PyTorch integration on top of the binding: an autograd function whose
forward is one ndvm_grad replay (loss and exact gradient of every lane in one
launch) and a calibration loop in which Adam (ndvm_adam_step) drives
ndvm_grad with the tape uploaded once, as in the paper's Kalman
maximum-likelihood fit (Section "From buckets to phases"); and autograd
functions of the encoder operators, for networks whose output is the replay's
parameters.  All arithmetic of
the replay and of the optimiser runs in the library's kernels; torch supplies
device memory and streams (and, for autograd, the chain rule of the caller's
own graph)."""
from __future__ import annotations

import torch
from torch.autograd.function import once_differentiable

from . import Tape, _launch_stream, _row_stride, adam_step, gated_ffn_grad, grad, layer_norm_grad, linear_attention_grad
from . import gated_ffn as gated_ffn_op
from . import layer_norm as layer_norm_op
from . import linear_attention as linear_attention_op


class ReplayLoss(torch.autograd.Function):
    """loss[L] = E(P, params[l]) per lane; backward scales each lane's exact
    gradient (computed in the forward replay) by the incoming loss gradient."""

    @staticmethod
    def forward(ctx, params, tape: Tape, obs, workspace=None):
        loss, g = grad(tape, params.detach(), obs, workspace=workspace)
        ctx.save_for_backward(g)
        return loss

    @staticmethod
    def backward(ctx, g_loss):
        (g,) = ctx.saved_tensors
        return g_loss.unsqueeze(1) * g, None, None, None


def replay_loss(tape: Tape, params, obs, workspace=None):
    """Per-lane loss with autograd support (see ReplayLoss)."""
    return ReplayLoss.apply(params, tape, obs, workspace)


def calibrate(tape: Tape, params, obs, steps: int, lr: float, beta1: float = 0.9, beta2: float = 0.999,
              eps: float = 1e-8, workspace=None, stream=None):
    """Fit every lane's parameters with `steps` Adam steps, in place.
    Returns the loss of every lane before each step, [steps, L]."""
    L, P = params.shape
    dev = params.device
    s = _launch_stream(stream, dev)
    # moments and buffers are allocated and zeroed on the stream the replay
    # and the optimiser steps run on, so the fills are ordered before them
    with torch.cuda.stream(s):
        m = torch.zeros((L, P), dtype=torch.float64, device=dev)
        v = torch.zeros((L, P), dtype=torch.float64, device=dev)
        g = torch.empty((L, P), dtype=torch.float64, device=dev)
        hist = torch.empty((steps, L), dtype=torch.float64, device=dev)
        for t in range(1, steps + 1):
            grad(tape, params, obs, loss=hist[t - 1], grad_out=g, workspace=workspace, stream=s)
            adam_step(params, g, m, v, t, lr, beta1, beta2, eps, stream=s)
    return hist


# ---------------------------------------------------------------- encoder operators
def _rows(x):
    """x, or a copy of it where its rows are not contiguous or do not lie at one stride."""
    try:
        _row_stride(x, "x")
    except ValueError:
        return x.contiguous()
    return x


class LayerNorm(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, bias, eps):
        x = _rows(x.detach())
        y, mean, rstd = layer_norm_op(x, weight, bias, eps)
        ctx.save_for_backward(x, weight, mean, rstd)
        ctx.has_bias = bias is not None
        return y

    @staticmethod
    @once_differentiable
    def backward(ctx, dy):
        x, weight, mean, rstd = ctx.saved_tensors
        need_weight = ctx.needs_input_grad[1] or ctx.needs_input_grad[2]
        dx, dw, db = layer_norm_grad(dy.contiguous(), x, weight, mean, rstd, ctx.needs_input_grad[0], need_weight)
        return dx, dw if ctx.needs_input_grad[1] else None, db if ctx.needs_input_grad[2] else None, None


def layer_norm(x, weight=None, bias=None, eps: float = 1e-5):
    """Layer norm over the last axis with autograd support (layer_norm of the package)."""
    return LayerNorm.apply(x, weight, bias, eps)


class LinearAttention(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, v, log_decay, offsets, scale, initial_state):
        o, last = linear_attention_op(q.detach(), k.detach(), v.detach(), log_decay, offsets, scale,
                                      None if initial_state is None else initial_state.detach(), final_state=True)
        ctx.save_for_backward(q, k, v, log_decay, offsets, initial_state)
        ctx.scale = scale
        ctx.set_materialize_grads(False)
        return o, last

    @staticmethod
    @once_differentiable
    def backward(ctx, do, dlast):
        q, k, v, log_decay, offsets, s0 = ctx.saved_tensors
        if do is None:
            do = torch.zeros((*q.shape[:-1], v.shape[-1]), dtype=q.dtype, device=q.device)
        need = list(ctx.needs_input_grad[:3])
        need[2] = need[2] or ctx.needs_input_grad[6]        # the state's gradient comes with v's
        dq, dk, dv, ds0 = linear_attention_grad(do.contiguous(), q, k, v, log_decay, offsets, ctx.scale, s0,
                                                None if dlast is None else dlast.contiguous(), tuple(need))
        return (dq, dk, dv if ctx.needs_input_grad[2] else None, None, None, None,
                ds0 if ctx.needs_input_grad[6] else None)


def linear_attention(q, k, v, log_decay, offsets=None, scale=None, initial_state=None):
    """(o, final state) with autograd support for q, k, v and the initial state
    (linear_attention of the package; the decay is a constant, and refused where it
    would need a gradient)."""
    if log_decay.requires_grad and torch.is_grad_enabled():
        raise ValueError("log_decay has no gradient: detach it")
    return LinearAttention.apply(q, k, v, log_decay, offsets, scale, initial_state)


class GatedFFN(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, w_gate, w_up, activation):
        x, w_gate, w_up = (_rows(t.detach()) for t in (x, w_gate, w_up))
        ctx.save_for_backward(x, w_gate, w_up)
        ctx.activation = activation
        return gated_ffn_op(x, w_gate, w_up, activation)

    @staticmethod
    @once_differentiable
    def backward(ctx, dh):
        x, w_gate, w_up = ctx.saved_tensors
        need_weight = ctx.needs_input_grad[1] or ctx.needs_input_grad[2]
        dx, dg, du = gated_ffn_grad(dh.contiguous(), x, w_gate, w_up, ctx.activation, ctx.needs_input_grad[0],
                                    need_weight)
        return dx, dg if ctx.needs_input_grad[1] else None, du if ctx.needs_input_grad[2] else None, None


def gated_ffn(x, w_gate, w_up, activation: str = "silu"):
    """act(x w_gate^T) * (x w_up^T) with autograd support (gated_ffn of the package)."""
    return GatedFFN.apply(x, w_gate, w_up, activation)

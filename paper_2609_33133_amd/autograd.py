"""Shared-prompt group attention as a differentiable torch op on one GPU.

    o_p, o_r = group_attention(q_p, k_p, v_p, q_r, k_r, v_r, batch)

Inputs are the packed bf16 tensors of a batch of replay trees (prompt rows
[T_P, H, d], response rows [T_R, H, d], `batch` the GroupBatch holding their
offsets). Forward: augtree_tree_fwd (the prompt, causal, once per tree, and
every branch against the prompt KV, read in place, plus its own causal KV; §3.2,
Eq. 1). Backward: augtree_tree_bwd (branch gradients, and the prompt-KV
gradient of every branch plus the prompt queries' own contribution summed on
the prompt KV in a fixed order, Eq. 2). Every step runs in the library's
kernels on the current stream; autograd only routes tensors. There is no CPU
path.

The layers of a model that keep a decayed state instead of a KV cache take the
same batches:

    o_p, o_r = group_linear_attention(q_p, k_p, v_p, q_r, k_r, v_r, batch, decay)
    y = head_norm(o_r, weight, bias, gate=gate, activation="silu")

The first computes a prompt's state once and goes on from it in every branch
(augtree_linear_fwd/bwd); the second is the norm over each head that follows
such a layer (augtree_head_norm_fwd/bwd). At decode, api.linear_step takes one
token of every sequence at a time.

A step, forward and backward, may be captured into a graph while no eager graph
of the same leaves is alive (torch's engine would join the two in the capture
and end the process).
"""
from __future__ import annotations

from typing import Optional, Tuple

import torch
from torch.autograd.function import once_differentiable

from . import api
from .api import REPLAY_FUSED, GroupBatch


def _check(t: torch.Tensor, name: str, rows: int, heads: int, d: int):
    if t.device.type != "cuda":
        raise ValueError(f"{name} must be a GPU tensor (the op has no CPU path)")
    if t.dtype != torch.bfloat16:
        raise TypeError(f"{name}: dtype {t.dtype}, expected torch.bfloat16")
    if tuple(t.shape) != (rows, heads, d):
        raise ValueError(f"{name}: shape {tuple(t.shape)}, expected {(rows, heads, d)}")


class _GroupAttention(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q_p, k_p, v_p, q_r, k_r, v_r, batch: GroupBatch, mode: int):
        b = batch
        for t, n, rows, h in ((q_p, "q_p", b.tp, b.hq), (k_p, "k_p", b.tp, b.hkv), (v_p, "v_p", b.tp, b.hkv),
                              (q_r, "q_r", b.tr, b.hq), (k_r, "k_r", b.tr, b.hkv), (v_r, "v_r", b.tr, b.hkv)):
            _check(t, n, rows, h, b.d)
        q_p, k_p, v_p, q_r, k_r, v_r = (t.contiguous() for t in (q_p, k_p, v_p, q_r, k_r, v_r))
        o_p, lse_p, o_r, lse_r = api.tree_fwd(b, q_p, k_p, v_p, q_r, k_r, v_r, mode)[:4]
        ctx.save_for_backward(q_p, k_p, v_p, q_r, k_r, v_r, o_p, lse_p, o_r, lse_r)
        ctx.batch = b
        ctx.mark_non_differentiable(lse_p, lse_r)
        return o_p, o_r

    @staticmethod
    def backward(ctx, do_p, do_r):
        b = ctx.batch
        q_p, k_p, v_p, q_r, k_r, v_r, o_p, lse_p, o_r, lse_r = ctx.saved_tensors
        # an output that did not reach the loss has a zero gradient
        do_p = torch.zeros_like(o_p) if do_p is None else do_p.to(torch.bfloat16).contiguous()
        do_r = torch.zeros_like(o_r) if do_r is None else do_r.to(torch.bfloat16).contiguous()
        dq_p, dk_p, dv_p, dq_r, dk_r, dv_r, _ = api.tree_bwd(b, q_p, k_p, v_p, o_p, lse_p, do_p, q_r, k_r, v_r, o_r,
                                                             lse_r, do_r)
        return dq_p, dk_p, dv_p, dq_r, dk_r, dv_r, None, None


def group_attention(q_p: torch.Tensor, k_p: torch.Tensor, v_p: torch.Tensor, q_r: torch.Tensor,
                    k_r: torch.Tensor, v_r: torch.Tensor, batch: GroupBatch,
                    mode: int = REPLAY_FUSED) -> Tuple[torch.Tensor, torch.Tensor]:
    """(O_P, O_R) of shared-prompt group attention; differentiable in all six inputs."""
    return _GroupAttention.apply(q_p, k_p, v_p, q_r, k_r, v_r, batch, int(mode))


def _trains(tensors) -> bool:
    """Whether a derivative may be asked for: otherwise autograd is left out, and its time. (A tangent counts, which the
    Functions refuse: it would get lost.)"""
    return (torch.is_grad_enabled() and any(t is not None and t.requires_grad for t in tensors)) or api._tangent(tensors)


class _GroupLinearAttention(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q_p, k_p, v_p, q_r, k_r, v_r, batch: GroupBatch, decay, state, return_state: bool):
        b = batch
        x = [t.contiguous() for t in (q_p, k_p, v_p, q_r, k_r, v_r)]
        ws = torch.empty(api.linear_workspace_size(b), dtype=torch.uint8, device=q_p.device)
        o_p, o_r, state_p, state_r = api.linear_fwd(b, decay, *x, state=state, want_states=return_state, ws=ws)
        ctx.save_for_backward(*x, ws)  # the backward takes its states from ws: the caller may go on with `state`
        ctx.batch, ctx.decay, ctx.ws_bytes = b, decay, api.linear_workspace_size(b, True, from_fwd_ws=True)
        ctx.set_materialize_grads(False)  # no zeros for the states' gradients, which nobody reads
        if not return_state:
            return o_p, o_r
        ctx.mark_non_differentiable(state_p, state_r)
        return o_p, o_r, state_p, state_r

    @staticmethod
    @once_differentiable
    def backward(ctx, do_p, do_r, *_):
        q_p, k_p, v_p, q_r, k_r, v_r, ws = ctx.saved_tensors
        # the forward has checked what it saved, autograd the gradients' shapes and device (None for an unused output)
        do_p, do_r = (torch.zeros_like(q) if g is None else g.to(torch.bfloat16).contiguous()
                      for g, q in ((do_p, q_p), (do_r, q_r)))
        with api._On((("q_p", q_p),)) as stream:
            grads = [torch.empty_like(t) for t in (q_p, k_p, v_p, q_r, k_r, v_r)]
            bwd_ws = torch.empty(ctx.ws_bytes, dtype=torch.uint8, device=q_p.device)
            api._linear_bwd(ctx.batch, ctx.decay, (q_p, k_p, v_p, do_p, q_r, k_r, v_r, do_r, None, *grads), ws, bwd_ws,
                            stream)
        return (*grads, None, None, None, None)


def group_linear_attention(q_p: torch.Tensor, k_p: torch.Tensor, v_p: torch.Tensor, q_r: torch.Tensor,
                           k_r: torch.Tensor, v_r: torch.Tensor, batch: GroupBatch, decay,
                           state: Optional[torch.Tensor] = None, return_state: bool = False):
    """(O_P, O_R) of linear attention over replay trees with a decay per KV head (host values in (0, 1]);
    differentiable in the six tensors. `state` [num_groups, Hkv, d, d] fp32 is what the prompts begin from; with
    `return_state` the states after every prompt and every branch follow the outputs (no gradient flows through
    either: a state, or a decay tensor, that asks for one is refused while gradients are enabled)."""
    if state is not None and state.requires_grad and torch.is_grad_enabled():
        raise ValueError("state is a constant of the op: no gradient is formed for it")
    decay = api._decay(decay, batch.hkv)
    x = (q_p, k_p, v_p, q_r, k_r, v_r)
    if not _trains(x + (state,)):
        out = api.linear_fwd(batch, decay, *(t.contiguous() for t in x), state=state, want_states=return_state)
        return out if return_state else out[:2]
    return _GroupLinearAttention.apply(*x, batch, decay.copy(), state, bool(return_state))


ACTIVATIONS = {"none": api.ACT_NONE, "silu": api.ACT_SILU}


class _HeadNorm(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, bias, gate, activation: int, eps: float):
        y = api.head_norm_fwd(x, weight, bias, gate, activation, eps)
        ctx.save_for_backward(x, weight, bias, gate)
        ctx.activation, ctx.eps = activation, eps
        return y

    @staticmethod
    @once_differentiable
    def backward(ctx, dy):
        x, weight, bias, gate = ctx.saved_tensors
        # the forward has checked what it saved, autograd the gradient's shape and device
        dy = dy.to(torch.bfloat16).contiguous()
        with api._On((("x", x),)) as stream:
            dx = torch.empty_like(x)
            dgate = None if gate is None else torch.empty_like(gate)
            dweight = torch.empty_like(weight) if ctx.needs_input_grad[1] else None
            dbias = torch.empty_like(bias) if ctx.needs_input_grad[2] else None
            api._head_norm_bwd(x, dy, weight, bias, gate, ctx.activation, ctx.eps, dx, dgate, dweight, dbias, None,
                               stream)
        return dx, dweight, dbias, dgate, None, None


def head_norm(x: torch.Tensor, weight: Optional[torch.Tensor] = None, bias: Optional[torch.Tensor] = None,
              gate: Optional[torch.Tensor] = None, activation: str = "none", eps: float = 1e-5) -> torch.Tensor:
    """Norm over each head of packed rows [rows, heads, head_dim] (bf16), n = (x - mean) / sqrt(var + eps), then
    a = n * weight + bias ([heads, head_dim] fp32, each optional) and y = act(a), or with a gate y = a * act(gate).
    `activation`: "none" or "silu". Differentiable in every tensor."""
    act = ACTIVATIONS.get(activation)
    if act is None:
        raise ValueError(f"activation {activation!r} not in {tuple(ACTIVATIONS)}")
    t = [None if v is None else v.contiguous() for v in (x, weight, bias, gate)]
    if not _trains(t):
        return api.head_norm_fwd(*t, act, eps)
    return _HeadNorm.apply(*t, act, float(eps))

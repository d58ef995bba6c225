"""One attention layer as it is trained with soft groups: the chain from the hidden states to the output, and back to the router's weights.

    forward    focus_router_scores (S = W_g h . C), focus_sinkhorn (soft assignments g), focus_gate_attn_fwd (o, lse)
    backward   focus_gate_attn_bwd (dq, dk, dv, dg), focus_sinkhorn_bwd (dg -> dS), focus_router_scores_bwd (dS -> dh, dW_g, dC)
    clip       focus_grad_clip over any gradients, the layer's own among them

A ``GateLayer`` holds what lies between the calls (scores, assignments, lse, their gradients) and one scratch buffer that the calls of a pass
use after one another, allocated once: ``forward``, ``backward`` and ``clip`` only enqueue, on the current stream (or ``stream``), and can be captured
into a graph.  A layer is for one stream at a time, and for one forward pass and its backward pass after it.  Its ``status`` says
whether a bounded wait of the attention ran out (``binding``'s status array; zeros otherwise).
"""
from __future__ import annotations

import torch

from . import binding as fb


class GateLayer:
    """``window``, ``scale``: as in ``binding.make_shape``; ``lam``: the gate's slope; ``tau``, ``iters``: of the Sinkhorn steps."""

    def __init__(self, batch, Hq, Hkv, n, D, K, d_model, d_g, window, lam, tau=0.1, iters=10, scale=0.0, device="cuda"):
        self.shape = fb.make_shape(Hq, Hkv, n, D, K, 1, window, scale, batch=batch)
        self.lam, self.tau, self.iters = lam, tau, iters
        sizes = [fb.focus_sinkhorn_workspace_bytes(self.shape, iters), fb.focus_sinkhorn_bwd_workspace_bytes(self.shape, iters),
                 fb.focus_gate_attn_bwd_workspace_bytes(self.shape), fb.focus_router_scores_bwd_workspace_bytes(self.shape, d_model, d_g)]
        if 0 in sizes:
            raise fb.FocusError(-1, fb.lib().focus_last_error().decode())
        f32 = dict(dtype=torch.float32, device=device)
        self.ws = torch.empty(max(sizes), dtype=torch.uint8, device=device)
        self.ws_clip = torch.empty(fb.focus_grad_clip_workspace_bytes(), dtype=torch.uint8, device=device)
        self.folded = torch.empty((K, d_model), **f32)
        self.scores, self.g, self.dg = (torch.empty((batch, n, fb.focus_soft_ld(K)), **f32) for _ in range(3))
        self.lse = torch.empty((batch, Hq, n), **f32)
        self.dWg, self.dC, self.norm = torch.empty((d_model, d_g), **f32), torch.empty((K, d_g), **f32), torch.empty(1, **f32)
        self.status = torch.zeros(4, dtype=torch.int32, device=device)

    def forward(self, h, q, k, v, Wg, C, o, stream=None):
        """h bf16 [batch, n, d_model]; q, o bf16 [batch, Hq, n, D]; k, v bf16 [batch, Hkv, n, D]; Wg fp32 [d_model, d_g], C fp32 [K, d_g].  Writes o."""
        fb.focus_router_scores(self.shape, h, Wg, C, self.folded, self.scores, stream)
        fb.focus_sinkhorn(self.shape, self.scores, self.tau, self.iters, self.ws, self.g, stream)
        fb.focus_gate_attn_fwd(self.shape, q, k, v, self.g, self.lam, o, self.lse, self.status, stream)

    def backward(self, h, q, k, v, Wg, C, o, d_o, dq, dk, dv, dh=None, stream=None):
        """The forward pass's tensors, as they were, and d_o like o.  Writes dq, dk, dv, ``self.dWg``, ``self.dC`` and, if given, dh: what goes to the
        hidden states by way of the router (that by way of q, k and v is the caller's to add)."""
        fb.focus_gate_attn_bwd(self.shape, q, k, v, self.g, self.lam, o, self.lse, d_o, dq, dk, dv, self.dg, self.ws, self.status, stream)
        fb.focus_sinkhorn_bwd(self.shape, self.scores, self.tau, self.iters, self.ws, self.dg, self.dg, stream)
        fb.focus_router_scores_bwd(self.shape, h, Wg, C, self.dg, dh, self.dWg, self.dC, self.ws, stream)

    def clip(self, grads, max_norm, stream=None):
        """Scales the gradients (``binding.make_grad_list``) so that their norm is at most ``max_norm``; the norm before goes to ``self.norm``."""
        fb.focus_grad_clip(grads, max_norm, self.norm, self.ws_clip, stream)

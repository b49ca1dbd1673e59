"""Attention over walks as a differentiable torch operation.

`attention` calls gs_attention_forward and, when gradients are asked for, gs_attention_backward
(include/gs.h).  `walk_lengths` gives the number of valid positions of the walks that
gs_random_walks / gs_node2vec_walks return, which is what the operation's lengths are made from.
"""
from __future__ import annotations

import torch

from . import binding as B


class _Gradient(torch.autograd.Function):
    """The gradients as a function of what they are computed from.  Under create_graph=True this node stands in the graph
    between them and the inputs, so that a second derivative meets an error here and does not take them for constants."""

    @staticmethod
    def forward(ctx, dout, q, k, v, out, lse, scale, window, q_lens, k_lens):
        return B.gs_attention_backward(dout, q, k, v, out, lse, scale, window, q_lens, k_lens)

    @staticmethod
    def backward(ctx, *grads):
        raise RuntimeError("attention is differentiable once: its gradients have no gradient")


class _Attention(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, v, scale, window, q_lens, k_lens):
        out, lse = B.gs_attention_forward(q, k, v, scale, window, q_lens, k_lens)
        ctx.save_for_backward(q, k, v, out, lse, q_lens, k_lens)
        ctx.scale, ctx.window = scale, window
        return out

    @staticmethod
    def backward(ctx, dout):
        q, k, v, out, lse, q_lens, k_lens = ctx.saved_tensors
        if dout.shape[3] > 1 and dout.stride(3) != 1:
            dout = dout.contiguous()
        gradient = _Gradient.apply if torch.is_grad_enabled() else B.gs_attention_backward
        dq, dk, dv = gradient(dout, q, k, v, out.detach(), lse, ctx.scale, ctx.window, q_lens, k_lens)
        return dq, dk, dv, None, None, None, None


def attention(q, k, v, scale=None, window=(-1, -1), q_lens=None, k_lens=None):
    """Attention of q[batch, q_len, q_heads, head_dim] over k, v[batch, k_len, kv_heads, head_dim];
    see gs_attention_forward in gs.h for the visible keys.  Differentiable once in q, k and v: a second
    derivative through it raises."""
    return _Attention.apply(q, k, v, scale, window, q_lens, k_lens)


def walk_lengths(walks: torch.Tensor) -> torch.Tensor:
    """Valid positions of each walk (int32[n_walks]): a walk is padded with -1 after its dead end."""
    return (walks >= 0).sum(dim=1, dtype=torch.int32)

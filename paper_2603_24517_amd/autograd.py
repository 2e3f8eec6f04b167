"""The operators of this package as torch.autograd sees them: functions of the same names and arguments whose results carry a
gradient.

    from paper_2603_24517_amd import autograd as AG
    q, k, v = AG.qkv_norm_rope(qkv, 32, 8, q_weight, k_weight, cos, sin)     # qkv [B, S, 32 + 8 + 8, 128], one projection
    o, lse = AG.attention(q, k, v, causal=True)

Gradients are those of include/attn_layer.h: not differentiable a second time, and not with respect to cos, sin and positions.  What is saved for the
backward pass are inputs and, of attention, O and LSE.  Forward and backward may be captured into a HIP graph together (torch's
rules for that hold: among them that no other autograd graph of the same leaves is alive while a backward pass is captured)."""
import torch
from torch.autograd.function import once_differentiable

import paper_2603_24517_amd as _attn


class _Attention(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, v, causal, scale):
        o, lse = _attn.attention(q, k, v, causal, scale)
        ctx.save_for_backward(q, k, v, o, lse)
        ctx.causal, ctx.scale = causal, scale
        ctx.set_materialize_grads(False)
        return o, lse

    @staticmethod
    @once_differentiable
    def backward(ctx, do, dlse):
        if do is None and dlse is None:
            return None, None, None, None, None
        q, k, v, o, lse = ctx.saved_tensors
        do = torch.zeros_like(q) if do is None else _whole(do)
        dlse = None if dlse is None else dlse.contiguous()
        return (*_attn.attention_backward(do, q, k, v, o, lse, ctx.causal, ctx.scale, dlse), None, None)


def attention(q, k, v, causal=False, scale=None):
    """attention(q, k, v, causal, scale) of the package; O and LSE both carry a gradient."""
    return _Attention.apply(q, k, v, causal, scale)


class _NormRope(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, v, q_weight, k_weight, cos, sin, positions, eps, interleaved):
        out = _attn.qk_norm_rope(q, k, q_weight, k_weight, cos, sin, positions, eps, interleaved, v)
        ctx.save_for_backward(q, k, q_weight, k_weight, cos, sin, positions)
        ctx.eps, ctx.interleaved = eps, interleaved
        ctx.set_materialize_grads(False)
        return out

    @staticmethod
    @once_differentiable
    def backward(ctx, dq, dk, dv=None):
        q, k, q_weight, k_weight, cos, sin, positions = ctx.saved_tensors
        dqw = dkw = None
        if dq is None and dk is None:
            return None, None, dv, None, None, None, None, None, None, None
        dq = torch.zeros(q.shape, dtype=q.dtype, device=q.device) if dq is None else _last(dq)
        dk = torch.zeros(k.shape, dtype=k.dtype, device=k.device) if dk is None else _last(dk)
        dq, dk, dqw, dkw = _attn.qk_norm_rope_backward(dq, dk, q, k, q_weight, k_weight, cos, sin, positions, ctx.eps, ctx.interleaved)
        return dq, dk, dv, _as(dqw, q_weight), _as(dkw, k_weight), None, None, None, None, None


class _FusedNormRope(torch.autograd.Function):
    @staticmethod
    def forward(ctx, qkv, heads, kv_heads, q_weight, k_weight, cos, sin, positions, eps, interleaved):
        q, k, v = qkv.split([heads, kv_heads, kv_heads], dim=2)
        out = _attn.qk_norm_rope(q, k, q_weight, k_weight, cos, sin, positions, eps, interleaved, v)
        ctx.save_for_backward(qkv, q_weight, k_weight, cos, sin, positions)
        ctx.heads, ctx.kv_heads, ctx.eps, ctx.interleaved = heads, kv_heads, eps, interleaved
        return out

    @staticmethod
    @once_differentiable
    def backward(ctx, dq, dk, dv):
        qkv, q_weight, k_weight, cos, sin, positions = ctx.saved_tensors
        parts = [ctx.heads, ctx.kv_heads, ctx.kv_heads]
        q, k, _ = qkv.split(parts, dim=2)
        dqkv = torch.empty(qkv.shape, dtype=qkv.dtype, device=qkv.device)
        *_, dqw, dkw = _attn.qk_norm_rope_backward(_last(dq), _last(dk), q, k, q_weight, k_weight, cos, sin, positions, ctx.eps, ctx.interleaved,
                                                   dv=_last(dv), out=dqkv.split(parts, dim=2))
        return dqkv, None, None, _as(dqw, q_weight), _as(dkw, k_weight), None, None, None, None, None


def _whole(g):
    """A contiguous gradient on a 16-byte boundary (a view into a larger one may be contiguous and off it)."""
    return g.contiguous() if not g.is_contiguous() else g if g.data_ptr() % 16 == 0 else g.clone()


def _last(g):
    """A gradient with strides that the kernels take: its last dimension contiguous, the others multiples of 8 elements, from 16 bytes on."""
    ok = g.stride(3) == 1 and all(n == 1 or s % 8 == 0 for n, s in zip(g.shape[:3], g.stride())) and g.data_ptr() % 16 == 0
    return g if ok else _whole(g)


def _as(gradient, weight):
    return None if gradient is None else gradient.to(weight.dtype)


def qk_norm_rope(q, k, q_weight, k_weight, cos, sin, positions=None, eps=1e-6, interleaved=False, v=None):
    """qk_norm_rope() of the package: (q, k), or (q, k, v) with v copied, with gradients of q, k, v and the weights."""
    return _NormRope.apply(q, k, v, q_weight, k_weight, cos, sin, positions, eps, interleaved)


def qkv_norm_rope(qkv, heads, kv_heads, q_weight, k_weight, cos, sin, positions=None, eps=1e-6, interleaved=False):
    """qk_norm_rope() on one projection qkv [B, S, heads + 2 * kv_heads, D]: contiguous q, k and v, as attention() takes them, in one
    pass; its gradient too is one pass and one tensor."""
    if qkv.dim() != 4 or qkv.shape[2] != heads + 2 * kv_heads:
        raise ValueError("qkv must be [B, S, heads + 2 * kv_heads, D]")
    return _FusedNormRope.apply(qkv, heads, kv_heads, q_weight, k_weight, cos, sin, positions, eps, interleaved)

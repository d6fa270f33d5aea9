"""Layers with gradients: LayerNorm, dropout and differential attention as
differentiable functions over the C ABI, and a window-attention Transformer
block built from them.

The inference modules approximate the attention of a trained model; this block
is what a model with differential attention (the difference of two softmax
maps over the same values, with a learned weight per head) is trained with.
Every step between the linear layers runs in the HIP library; the linear layers
and GELU are torch's.

Recording a graph: the functions refuse to take part in one when gradients are
asked for.  Their backward pass would accumulate into leaves that an eager
graph may still hold on another stream, which ends the process; a training
step is recorded with the explicit calls (``binding.nystra_*_backward``).
"""

import torch
from torch import nn
from torch.autograd.function import once_differentiable

from . import binding as B


def _differentiated(*tensors):
    """Whether a backward pass may follow: without one nothing is kept for it."""
    return torch.is_grad_enabled() and any(t is not None and t.requires_grad for t in tensors)


def _not_recorded(*tensors):
    if _differentiated(*tensors) and torch.cuda.is_current_stream_capturing():
        raise RuntimeError("gradients in a recorded graph: call the binding's forward and "
                           "backward entry points instead")


def _not_recorded_backward():
    if torch.cuda.is_current_stream_capturing():
        raise RuntimeError("the backward pass of these functions cannot be recorded: call the "
                           "binding's backward entry points instead")


class _LayerNorm(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, bias, eps, keep):
        if not keep:
            return B.nystra_layer_norm_forward(x, weight, bias, eps)
        y, mean, rstd = B.nystra_layer_norm_forward(x, weight, bias, eps, with_stats=True)
        ctx.save_for_backward(x, weight, mean, rstd)
        return y

    @staticmethod
    @once_differentiable
    def backward(ctx, dy):
        _not_recorded_backward()
        x, weight, mean, rstd = ctx.saved_tensors
        dx, dw, db = B.nystra_layer_norm_backward(dy.contiguous(), x, weight, mean, rstd)
        need = ctx.needs_input_grad
        return dx, dw if need[1] else None, db if need[2] else None, None, None


class _Dropout(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, residual, p, seed, offset):
        ctx.args = p, seed, offset
        return B.nystra_dropout(x, p, seed, offset, residual=residual)

    @staticmethod
    @once_differentiable
    def backward(ctx, dy):
        _not_recorded_backward()
        need = ctx.needs_input_grad
        dx = B.nystra_dropout(dy.contiguous(), *ctx.args) if need[0] else None
        return dx, dy if need[1] else None, None, None, None


class _DiffAttention(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, v, lam, scale, causal, kv_len, keep):
        o = B.nystra_diff_attn_forward(q, k, v, lam, scale=scale, causal=causal, kv_len=kv_len,
                                       with_saved=keep)
        if not keep:
            return o
        o, saved = o
        ctx.save_for_backward(q, k, v, lam, o, kv_len, *saved)
        ctx.args = dict(scale=scale, causal=causal)
        return o

    @staticmethod
    @once_differentiable
    def backward(ctx, do):
        _not_recorded_backward()
        q, k, v, lam, o, kv_len, maps, sums = ctx.saved_tensors
        grads = B.nystra_diff_attn_backward(do.contiguous(), q, k, v, lam, o, (maps, sums),
                                            kv_len=kv_len, **ctx.args)
        return (*grads, None, None, None, None)


def _packed_views(qkv, heads):
    """Q, K [W, 2 heads, N, C / 2 heads] and V [W, heads, N, C / heads] of a projection's
    output [W, N, 3 C], as it lies."""
    q, k, v = qkv.chunk(3, dim=-1)
    return (q.unflatten(-1, (2 * heads, -1)).transpose(1, 2),
            k.unflatten(-1, (2 * heads, -1)).transpose(1, 2),
            v.unflatten(-1, (heads, -1)).transpose(1, 2))


class _PackedDiffAttention(torch.autograd.Function):
    """On the projection's output, whose gradient is written as one tensor."""

    @staticmethod
    def forward(ctx, qkv, lam, heads, keep):
        W, N, C3 = qkv.shape
        out = qkv.new_empty(W, N, heads, C3 // 3 // heads)
        got = B.nystra_diff_attn_forward(*_packed_views(qkv, heads), lam, with_saved=keep,
                                         out=out.transpose(1, 2))
        if keep:
            ctx.save_for_backward(qkv, lam, out, *got[1])
        return out

    @staticmethod
    @once_differentiable
    def backward(ctx, do):
        _not_recorded_backward()
        qkv, lam, out, maps, sums = ctx.saved_tensors
        heads = out.shape[2]
        grad = torch.empty_like(qkv)
        *_, dlam = B.nystra_diff_attn_backward(
            do.contiguous().transpose(1, 2), *_packed_views(qkv, heads), lam,
            out.transpose(1, 2), (maps, sums), grads=_packed_views(grad, heads))
        return grad, dlam, None, None


def _row_strided(x):
    """Whether x [..., C] is a list of rows at one stride, none of them over another."""
    try:
        return B._rows(x, x.shape[-1]) >= x.shape[-1]
    except (IndexError, ValueError):
        return False


def layer_norm(x, weight=None, bias=None, eps=1e-5):
    """LayerNorm over the last dimension, differentiable in x, weight and bias.  Weights of
    another type are rounded to x's, half a step of it relative to each, as a layer of that
    type holds them; their gradients come in their own.  Rows that do not lie at one stride
    are copied."""
    _not_recorded(x, weight, bias)
    if not _row_strided(x):
        x = x.contiguous()
    weight, bias = (None if t is None else t.to(x.dtype) for t in (weight, bias))
    return _LayerNorm.apply(x, weight, bias, eps, _differentiated(x, weight, bias))


def dropout(x, p, seed, offset=0, residual=None):
    """residual + dropout(x), differentiable in both; the mask is a function of seed and
    offset and is formed again in the backward pass.  Of two types the sum is of the wider
    one: a bf16 branch leaves an fp32 residual stream in fp32."""
    _not_recorded(x, residual)
    if residual is not None:
        dtype = torch.promote_types(x.dtype, residual.dtype)
        x, residual = x.to(dtype), residual.to(dtype).contiguous()
    return _Dropout.apply(x.contiguous(), residual, p, seed, offset)


def differential_attention(q, k, v, lam, scale=0.0, causal=B.CAUSAL_NONE, kv_len=None):
    """binding.nystra_diff_attn_forward, differentiable in q, k, v and lam (of any type: it
    counts in fp32)."""
    _not_recorded(q, k, v, lam)
    lam = lam.float()
    return _DiffAttention.apply(q, k, v, lam, scale, causal, kv_len,
                                _differentiated(q, k, v, lam))


class LayerNorm(nn.LayerNorm):
    """nn.LayerNorm over the last dimension, by the library's kernels."""

    def __init__(self, channels, eps=1e-5, **kw):
        super().__init__(channels, eps=eps, **kw)
        if (len(self.normalized_shape) != 1 or
                not 1 <= self.normalized_shape[0] <= B.NORM_MAX_CHANNELS):
            raise ValueError(f"expected one dimension of 1 to {B.NORM_MAX_CHANNELS} channels")

    def forward(self, x):
        return layer_norm(x, self.weight, self.bias, self.eps)


class DifferentialWindowAttention(nn.Module):
    """Window attention with two softmax maps per head on x [B, H, W, C]:
    (softmax(Q1 K1^T) - lam softmax(Q2 K2^T)) V in every window, LayerNorm of each head's
    output, and the output projection.  lam follows from learned vectors per head,
    lam = exp(a1 . b1) - exp(a2 . b2) + lam_init."""

    def __init__(self, dim, heads, window, shift=0, lam_init=0.8, dtype=torch.float32,
                 device="cuda"):
        super().__init__()
        if dim % (2 * heads) != 0:
            raise ValueError("2 heads must divide dim")
        if dim // (2 * heads) > B.DIFF_MAX_WIDTH:
            raise ValueError(f"heads of more than {B.DIFF_MAX_WIDTH} channels to a map")
        if not 0 <= shift < window:
            raise ValueError("shift must be in [0, window)")
        kw = dict(dtype=dtype, device=device)
        self.dim, self.heads, self.window, self.shift = dim, heads, window, shift
        self.lam_init = lam_init
        self.qkv = nn.Linear(dim, 3 * dim, **kw)
        self.proj = nn.Linear(dim, dim, **kw)
        self.norm = LayerNorm(dim // heads, **kw)
        # fp32 whatever the layer's type, and formed in fp32 also where the module was moved to
        # another one: lam is the difference of two exponentials.
        self.lam = nn.Parameter(0.1 * torch.randn(4, heads, dim // (2 * heads), device=device))

    def weights(self):
        """lam, fp32 [heads]."""
        a1, b1, a2, b2 = self.lam.float()
        return torch.exp((a1 * b1).sum(-1)) - torch.exp((a2 * b2).sum(-1)) + self.lam_init

    def forward(self, x):
        Bn, H, W, C = x.shape
        w = self.window
        if C != self.dim or H % w != 0 or W % w != 0:
            raise ValueError(f"expected [B, H, W, {self.dim}] with {w} dividing H and W")
        if self.shift:
            x = x.roll((-self.shift, -self.shift), (1, 2))
        win = x.view(Bn, H // w, w, W // w, w, C).transpose(2, 3).reshape(-1, w * w, C)
        qkv, lam = self.qkv(win), self.weights()
        _not_recorded(qkv, lam)
        # [windows, N, heads, C / heads]
        o = _PackedDiffAttention.apply(qkv, lam, self.heads, _differentiated(qkv, lam))
        o = self.norm(o) * (1.0 - self.lam_init)
        y = self.proj(o.flatten(2))
        y = y.view(Bn, H // w, W // w, w, w, C).transpose(2, 3).reshape(Bn, H, W, C)
        return y.roll((self.shift, self.shift), (1, 2)) if self.shift else y


class DifferentialTransformerBlock(nn.Module):
    """x + dropout(attn(norm1(x))), then + dropout(mlp(norm2(.))), on x [B, H, W, C].

    In training every call draws one seed from torch's host generator (torch.manual_seed)
    for the masks of its two branches; ``seed`` may be given instead."""

    def __init__(self, dim, heads, window, shift=0, mlp_ratio=2.0, p=0.1, lam_init=0.8,
                 dtype=torch.float32, device="cuda"):
        super().__init__()
        if not 0 <= p <= 1:
            raise ValueError("p must be in [0, 1]")
        kw = dict(dtype=dtype, device=device)
        hidden = int(dim * mlp_ratio)
        self.p = p
        self.norm1 = LayerNorm(dim, **kw)
        self.attn = DifferentialWindowAttention(dim, heads, window, shift, lam_init, **kw)
        self.norm2 = LayerNorm(dim, **kw)
        self.mlp = nn.Sequential(nn.Linear(dim, hidden, **kw), nn.GELU(),
                                 nn.Linear(hidden, dim, **kw))

    def forward(self, x, seed=None):
        p = self.p if self.training else 0.0
        if seed is None:
            seed = int(torch.randint(1 << 62, (1,))) if p > 0 else 0
        x = dropout(self.attn(self.norm1(x.contiguous())), p, seed, 0, residual=x)
        return dropout(self.mlp(self.norm2(x)), p, seed, 1, residual=x)

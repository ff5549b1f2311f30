"""torch.autograd wrapper around the C ABI: argument marshalling only.

    from paper_2505_09326_amd.autograd import spherical_attention
    O = spherical_attention(Q, K, V)          # [B,H,N,d] bf16 or fp16 CUDA tensors
    O.sum().backward()                        # dQ, dK, dV from sphattn_bwd / sphattn_grn_bwd

    X = token_embedding(tokens, table, mult, scale)      # rows of a table, scaled
    loss = vocab_cross_entropy(X, W, targets)            # -log softmax(X W^T)[targets], no logits in memory

Forward = sphattn_fwd_z (O and the row aggregates z, which the backward needs), or
sphattn_cross_fwd when multiplicities or shared K/V heads are given; backward = the library's
two backward kernels.  Nothing is computed here.
"""
import math

import torch
from torch.autograd.function import once_differentiable

from . import (REDUCTIONS, _cross_fwd_z, _fast_calls, sphattn_bwd, sphattn_embed_bwd, sphattn_embed_fwd, sphattn_fwd_z, sphattn_grn_bwd,
               sphattn_vocab_loss_bwd, sphattn_vocab_loss_fwd)

_DTYPES = {torch.bfloat16: "bf16", torch.float16: "f16"}


class _SphericalAttention(torch.autograd.Function):
    @staticmethod
    def forward(ctx, Q, K, V, mult):
        if Q.dtype not in _DTYPES or K.dtype != Q.dtype or V.dtype != Q.dtype:
            raise TypeError("spherical_attention differentiates bf16 or fp16 tensors of one dtype")
        if Q.dim() != 4 or K.dim() != 4 or K.shape[2] != Q.shape[2]:
            # the backward kernels are self-attention only; catch it before anything is launched
            raise ValueError(f"spherical_attention needs K, V with Q's N: Q {tuple(Q.shape)}, K {tuple(K.shape)}")
        dtype = _DTYPES[Q.dtype]
        Q, K, V = Q.contiguous(), K.contiguous(), V.contiguous()
        plain = mult is None and K.shape[1] == Q.shape[1]
        O, Z = sphattn_fwd_z(Q, K, V, dtype=dtype) if plain else _cross_fwd_z(Q, K, V, mult, dtype)
        ctx.save_for_backward(Q, K, V, O, Z)
        ctx.mult, ctx.plain, ctx.dtype = mult, plain, dtype
        return O

    @staticmethod
    def backward(ctx, dO):
        Q, K, V, O, Z = ctx.saved_tensors
        dO = dO.contiguous()
        if ctx.plain:
            dQ, dK, dV = sphattn_bwd(Q, K, V, O, dO, Z, dtype=ctx.dtype)
        else:
            dQ, dK, dV = sphattn_grn_bwd(Q, K, V, ctx.mult, O, dO, Z, dtype=ctx.dtype)
        return dQ, dK, dV, None


def spherical_attention(Q, K, V, mult=None):
    """Differentiable spherical attention: Q [B,H,N,d]; K, V [B,H_kv,N,d]; optional per-key
    multiplicities mult [B,N] (fp32, no gradient)."""
    return _SphericalAttention.apply(Q, K, V, mult)


class _TokenEmbedding(torch.autograd.Function):
    @staticmethod
    def forward(ctx, tokens, table, mult, scale):
        shape, tokens = tokens.shape, tokens.reshape(-1).contiguous()
        if mult is not None:
            if mult.shape != shape:
                raise ValueError(f"mult must have the tokens' shape {tuple(shape)}, got {tuple(mult.shape)}")
            mult = mult.reshape(-1).contiguous()
        O = sphattn_embed_fwd(tokens, table.contiguous(), mult, scale)
        ctx.save_for_backward(tokens, mult)
        ctx.V, ctx.scale = table.shape[0], scale
        return O.view(*shape, O.shape[1])

    @staticmethod
    @once_differentiable
    def backward(ctx, dO):
        tokens, mult = ctx.saved_tensors
        return None, sphattn_embed_bwd(tokens, dO.reshape(-1, dO.shape[-1]).contiguous(), ctx.V, mult, ctx.scale), None, None


def token_embedding(tokens, table, mult=None, scale=1.0):
    """Differentiable embedding lookup with scaling, scale * mult * table[tokens]: tokens of any shape (int32 or int64; negative: no
    token, a row of zeros), table [V,D] (fp32, bf16 or fp16), mult of the tokens' shape (fp32, no gradient) or None."""
    done = _fast_calls().embed_forward(tokens, table, mult, scale, True)
    return _TokenEmbedding.apply(tokens, table, mult, scale) if done is None else done


class _VocabCrossEntropy(torch.autograd.Function):
    @staticmethod
    def forward(ctx, X, W, targets, scale, reduction):
        if X.dtype != W.dtype:
            raise TypeError(f"X and W must have one dtype, got {X.dtype} and {W.dtype}")
        if X.shape[:-1] != targets.shape:
            raise ValueError(f"targets must have the shape of X's rows {tuple(X.shape[:-1])}, got {tuple(targets.shape)}")
        ctx.shape, ctx.scale, ctx.reduction = X.shape, scale, reduction
        X, W, targets = X.reshape(-1, X.shape[-1]).contiguous(), W.contiguous(), targets.reshape(-1).contiguous()
        got = sphattn_vocab_loss_fwd(X, W, targets, scale, reduction, all_rows=False)
        ctx.save_for_backward(X, W, targets, got[1])
        return got[2] if reduction != "none" else got[0].view(ctx.shape[:-1])

    @staticmethod
    @once_differentiable
    def backward(ctx, dloss):
        X, W, targets, lse = ctx.saved_tensors
        if ctx.reduction == "none":
            dloss = dloss.reshape(-1)
        dX, dW = sphattn_vocab_loss_bwd(X, W, targets, lse, dloss.contiguous(), ctx.scale, ctx.reduction,
                                        want_dX=ctx.needs_input_grad[0], want_dW=ctx.needs_input_grad[1])
        return None if dX is None else dX.view(ctx.shape), dW, None, None, None


def vocab_cross_entropy(X, W, targets, scale=1.0, reduction="mean"):
    """Differentiable cross entropy of softmax(scale * X W^T) over a vocabulary, in fp32: X [..., D] and W [V,D] of one type (fp32, bf16 or
    fp16), targets [...] (int32 or int64; negative: the row does not count).  reduction "mean" (over the rows that count; 0 if
    none does), "sum" or "none"."""
    scale = float(scale)
    if math.isfinite(scale):                       # (else the Python path says so)
        done = _fast_calls().loss_forward(X, W, targets, scale, REDUCTIONS[reduction], False, True)
        if done is not None:
            return done
    return _VocabCrossEntropy.apply(X, W, targets, scale, reduction)

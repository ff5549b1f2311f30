"""torch.autograd wrapper around the C ABI: argument marshalling only.

    from paper_2505_09326_amd.autograd import spherical_attention
    O = spherical_attention(Q, K, V)          # [B,H,N,d] bf16 or fp16 CUDA tensors
    O.sum().backward()                        # dQ, dK, dV from sphattn_bwd / sphattn_grn_bwd

    X = token_embedding(tokens, table, mult, scale)      # rows of a table, scaled
    Q, K = head_norm_rotary(Xq, Xk, wq, wk, positions, inv_freq)      # norms of heads, rotated by positions, as the attention reads them
    H = gated_feed_forward(X, Wg, Wu)                    # silu(X Wg^T) * (X Wu^T)
    loss = vocab_cross_entropy(X, W, targets)            # -log softmax(X W^T)[targets], no logits in memory
    loss = vocab_distillation(X, W, ids, teacher)        # softmax(X W^T) against a teacher's best logits

Forward = sphattn_fwd_z (O and the row aggregates z, which the backward needs), or
sphattn_cross_fwd when multiplicities or shared K/V heads are given; backward = the library's
two backward kernels.  Nothing is computed here.
"""
import math

import torch
from torch.autograd.function import once_differentiable

from . import (GATES, REDUCTIONS, _cross_fwd_z, _fast_calls, sphattn_bwd, sphattn_embed_bwd, sphattn_embed_fwd, sphattn_fwd_z, sphattn_gated_ffn_bwd,
               sphattn_gated_ffn_fwd, sphattn_grn_bwd, sphattn_head_norm_rotary_bwd, sphattn_head_norm_rotary_fwd, sphattn_vocab_distill_bwd,
               sphattn_vocab_distill_fwd, sphattn_vocab_loss_bwd, sphattn_vocab_loss_fwd)

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


class _HeadNormRotary(torch.autograd.Function):
    @staticmethod
    def forward(ctx, Xq, Xk, wq, wk, positions, inv_freq, sections, interleaved, norm, eps):
        rows = lambda t: t if t is None or t.stride(-1) == 1 else t.contiguous()
        Xq, Xk, wq, wk = rows(Xq), rows(Xk), *(None if w is None else w.contiguous() for w in (wq, wk))
        ctx.rotary = (positions, inv_freq, sections, interleaved, norm, eps)
        Q, K = sphattn_head_norm_rotary_fwd(Xq, Xk, wq, wk, *ctx.rotary)
        ctx.save_for_backward(Xq, Xk, wq, wk, positions, inv_freq)
        ctx.rotary = (sections, interleaved, norm, eps)
        return Q, K

    @staticmethod
    @once_differentiable
    def backward(ctx, dQ, dK):
        Xq, Xk, wq, wk, positions, inv_freq = ctx.saved_tensors
        rows = lambda t: t if t is None or t.stride(-1) == 1 else t.contiguous()
        need = ctx.needs_input_grad
        grads = sphattn_head_norm_rotary_bwd(Xq, Xk, wq, wk, rows(dQ), rows(dK) if Xk is not None else None, positions, inv_freq, *ctx.rotary,
                                             want_dX=need[:2], want_dw=need[2:4])
        return *grads, None, None, None, None, None, None


def head_norm_rotary(Xq, Xk=None, wq=None, wk=None, positions=None, inv_freq=None, sections=None, interleaved=False, norm=True, eps=1e-6):
    """Differentiable norms of queries Xq [B,N,Hq,d] and keys Xk [B,N,Hk,d] (or None) for each head, times wq and wk [d], rotated by their
    positions, laid out for spherical_attention: (Q [B,Hq,N,d], K [B,Hk,N,d] or None).  Xq and Xk may be slices of one projection's
    output.  Arguments as sphattn_head_norm_rotary_fwd; no gradients of positions and inv_freq."""
    eps = float(eps)
    if math.isfinite(eps):                         # (else the Python path says so)
        done = _fast_calls().heads_forward(Xq, Xk, wq, wk, positions, inv_freq, sections, bool(interleaved), bool(norm), eps, None, None, True)
        if done is not None:
            return done
    return _HeadNormRotary.apply(Xq, Xk, wq, wk, positions, inv_freq, sections, interleaved, norm, eps)


class _GatedFeedForward(torch.autograd.Function):
    @staticmethod
    def forward(ctx, X, Wg, Wu, activation):
        if X.dtype != Wg.dtype or X.dtype != Wu.dtype:
            raise TypeError(f"X, Wg and Wu must have one dtype, got {X.dtype}, {Wg.dtype} and {Wu.dtype}")
        ctx.shape, ctx.activation = X.shape, activation
        X, Wg, Wu = X.reshape(-1, X.shape[-1]).contiguous(), Wg.contiguous(), Wu.contiguous()
        ctx.save_for_backward(X, Wg, Wu)
        return sphattn_gated_ffn_fwd(X, Wg, Wu, activation).view(*ctx.shape[:-1], Wg.shape[0])

    @staticmethod
    @once_differentiable
    def backward(ctx, dH):
        X, Wg, Wu = ctx.saved_tensors
        need = ctx.needs_input_grad
        dX, dWg, dWu = sphattn_gated_ffn_bwd(X, Wg, Wu, dH.reshape(-1, dH.shape[-1]).contiguous(), ctx.activation, want_dX=need[0], want_dWg=need[1],
                                             want_dWu=need[2])
        return None if dX is None else dX.view(ctx.shape), dWg, dWu, None


def gated_feed_forward(X, Wg, Wu, activation="silu"):
    """Differentiable act(X Wg^T) * (X Wu^T): X [..., D], Wg and Wu [F,D] of one type (fp32, bf16 or fp16), activation "silu", "gelu" or "relu".  Nothing but
    the inputs is kept for the gradients."""
    done = _fast_calls().ffn_forward(X, Wg, Wu, GATES[activation], True)
    return done if done is not None else _GatedFeedForward.apply(X, Wg, Wu, activation)


class _VocabDistillation(torch.autograd.Function):
    @staticmethod
    def forward(ctx, X, W, ids, teacher, scale, temperature, reduction):
        if X.dtype != W.dtype:
            raise TypeError(f"X and W must have one dtype, got {X.dtype} and {W.dtype}")
        if ids.dim() < 1 or X.shape[:-1] != ids.shape[:-1] or teacher.shape != ids.shape:
            raise ValueError(f"ids and teacher must be [..., K] with X's rows {tuple(X.shape[:-1])}, got {tuple(ids.shape)} and {tuple(teacher.shape)}")
        ctx.shape, ctx.how = X.shape, (scale, temperature, reduction)
        X, W = X.reshape(-1, X.shape[-1]).contiguous(), W.contiguous()
        ids, teacher = (t.reshape(-1, t.shape[-1]).contiguous() for t in (ids, teacher))
        losses, lse, kept, *mean = sphattn_vocab_distill_fwd(X, W, ids, teacher, *ctx.how, keep=True)
        ctx.save_for_backward(X, W, ids, teacher, lse, kept)
        return mean[0] if mean else losses.view(ctx.shape[:-1])

    @staticmethod
    @once_differentiable
    def backward(ctx, dloss):
        X, W, ids, teacher, lse, kept = ctx.saved_tensors
        if ctx.how[2] == "none":
            dloss = dloss.reshape(-1)
        dX, dW = sphattn_vocab_distill_bwd(X, W, ids, teacher, lse, kept, dloss.contiguous(), *ctx.how, want_dX=ctx.needs_input_grad[0],
                                           want_dW=ctx.needs_input_grad[1])
        return None if dX is None else dX.view(ctx.shape), dW, None, None, None, None, None


def vocab_distillation(X, W, ids, teacher, scale=1.0, temperature=1.0, reduction="mean"):
    """Differentiable divergence of softmax(scale / temperature X W^T) over a vocabulary from a teacher's best logits, times temperature^2, in fp32: X [..., D]
    and W [V,D] of one type (fp32, bf16 or fp16), ids [..., K] (int32 or int64; negative: no entry), teacher [..., K] (fp32, its logits of those ids, no
    gradient).  reduction "mean" (over the rows with an entry; 0 if there is none), "sum" or "none"."""
    scale, temperature = float(scale), float(temperature)
    if math.isfinite(scale) and 2.0 ** -20 <= temperature <= 2.0 ** 20:      # (else the Python path says so)
        done = _fast_calls().distill_forward(X, W, ids, teacher, scale, temperature, REDUCTIONS[reduction], True, True)
        if done is not None:
            return done
    return _VocabDistillation.apply(X, W, ids, teacher, scale, temperature, reduction)

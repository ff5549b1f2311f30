#!/usr/bin/env python3
"""Training a small layer from a teacher's best answers on synthetic cells, everything but the plain projections from this package's kernels:

    python examples/distill_masked_genes.py [--steps 100]

A cell is a set of gene tokens with counts, each gene at a place of a chromosome.  For every token a teacher says which K genes it holds for likely there:

    X     = sqrt(D) * log(1 + count) * table[tokens]                       token_embedding
    Q, K  = norms of heads, rotated by (chromosome, place)                 head_norm_rotary
    X    += attention(Q, K, V) Wo, four query heads to a key head          spherical_attention
    X    += (silu(X Wg^T) * (X Wu^T)) Wd                                   gated_feed_forward
    loss  = divergence of softmax(X table^T) from the teacher's answers    vocab_distillation
    gradients scaled down to a common norm of at most 1                    sphattn_clip_grads

The teacher knows the cell's type and the genes that it expresses."""
import argparse
import math
import os
import sys

import torch

sys.path.insert(0, os.path.join(os.path.dirname(os.path.abspath(__file__)), ".."))

import paper_2505_09326_amd as sph
from paper_2505_09326_amd.autograd import gated_feed_forward, head_norm_rotary, spherical_attention, token_embedding, vocab_distillation

CHROMOSOMES, TEMPERATURE = 23, 2.0


def cells(batch, length, genes, types, best, generator, device):
    """tokens and counts [batch, length], the teacher's ids and logits [batch, length, best]: -1 where it has no more to say."""
    per_type = genes // types
    kind = torch.randint(types, (batch, 1), generator=generator, device=device)
    tokens = kind * per_type + torch.randint(per_type, (batch, length), generator=generator, device=device)
    counts = torch.poisson(torch.full((batch, length), 2.0, device=device), generator=generator) + 1
    first = torch.randint(per_type, (batch, length, 1), generator=generator, device=device)
    ids = kind[:, :, None] * per_type + (first + 7 * torch.arange(best, device=device)) % per_type
    teacher = 4.0 - 0.5 * torch.arange(best, device=device) + 0.3 * torch.randn((batch, length, best), generator=generator, device=device)
    said = torch.randint(best + 1, (batch, length, 1), generator=generator, device=device)
    return tokens, counts, torch.where(torch.arange(best, device=device) < said, ids, -1), teacher


def new_weights(genes, heads, key_heads, width, inner, generator, device, dtype=torch.bfloat16):
    """table, Wqkv, wq, wk, Wo, Wg, Wu, Wd"""
    D = heads * width
    new = lambda *shape, scale: (torch.randn(shape, generator=generator, device=device) * scale).to(dtype).requires_grad_(True)
    ones = lambda: torch.ones(width, device=device, dtype=dtype).requires_grad_(True)
    return [new(genes, D, scale=0.5 * D ** -0.5), new(D, (heads + 2 * key_heads) * width, scale=D ** -0.5), ones(), ones(), new(D, D, scale=D ** -0.5),
            new(inner, D, scale=D ** -0.5), new(inner, D, scale=D ** -0.5), new(inner, D, scale=inner ** -0.5)]


def frequencies(width, device):
    """inv_freq [width / 2], how many of them go by the chromosome and how many by the place"""
    sections = [width // 8, width // 2 - width // 8]
    return torch.cat([torch.pow(1000.0, -torch.arange(n, device=device, dtype=torch.float64) / n) for n in sections]).float(), sections


def student(weights, tokens, counts, heads, key_heads):
    """Hidden states [batch, length, D]."""
    table, Wqkv, wq, wk, Wo, Wg, Wu, Wd = weights
    (batch, length), D = tokens.shape, table.shape[1]
    width = D // heads
    inv_freq, sections = frequencies(width, tokens.device)
    X = token_embedding(tokens, table, torch.log1p(counts), math.sqrt(D))
    q, k, v = (X @ Wqkv).view(batch, length, -1, width).split([heads, key_heads, key_heads], 2)
    Q, K = head_norm_rotary(q, k, wq, wk, torch.stack([tokens % CHROMOSOMES, tokens // CHROMOSOMES]), inv_freq, sections)
    O = spherical_attention(Q, K, v.transpose(1, 2).contiguous())
    X = X + O.transpose(1, 2).reshape(batch, length, D) @ Wo
    return X + gated_feed_forward(X, Wg, Wu) @ Wd


def train(steps=100, batch=8, length=512, genes=4000, types=20, best=16, heads=4, key_heads=1, width=64, inner=512, lr=3e-3, device="cuda:0", seed=0):
    """Losses and gradient norms of the steps."""
    g = torch.Generator(device=device).manual_seed(seed)
    weights = new_weights(genes, heads, key_heads, width, inner, g, device)
    masters = [w.detach().float() for w in weights]            # (the steps are smaller than bf16's)
    optimizer = torch.optim.Adam(masters, lr=lr)
    losses, norms = [], []
    for _ in range(steps):
        tokens, counts, ids, teacher = cells(batch, length, genes, types, best, g, device)
        loss = vocab_distillation(student(weights, tokens, counts, heads, key_heads), weights[0], ids, teacher, temperature=TEMPERATURE)
        grads = list(torch.autograd.grad(loss, weights))
        norms.append(sph.sphattn_clip_grads(grads, 1.0))
        for m, d in zip(masters, grads):
            m.grad = d.float()
        optimizer.step()
        with torch.no_grad():
            for w, m in zip(weights, masters):
                w.copy_(m)
        losses.append(loss.detach())
    return torch.stack(losses).tolist(), torch.stack(norms).tolist()


if __name__ == "__main__":
    parser = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    parser.add_argument("--steps", type=int, default=100)
    got, norms = train(steps=parser.parse_args().steps)
    for i, (loss, norm) in enumerate(zip(got, norms)):
        print(f"step {i:3d}  loss {loss:.4f}  gradient norm {norm:.3f}")

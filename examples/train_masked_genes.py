#!/usr/bin/env python3
"""Masked-gene training of a one-layer model on synthetic cells, everything but the projections from this package's kernels:

    python examples/train_masked_genes.py [--steps 100]

A cell is a set of gene tokens with counts.  Some tokens are hidden; the model says which genes they were:

    X     = sqrt(D) * log(1 + count) * table[tokens]          token_embedding
    X    += attention(X Wq, X Wk, X Wv) Wo                    spherical_attention
    loss  = mean over the hidden tokens of -log softmax(X table^T)[gene]     vocab_cross_entropy (the table is the head, too)
    gradients scaled down to a common norm of at most 1       sphattn_clip_grads

Cells are of a few types that express genes of their own, so the genes in sight tell something about the hidden ones: the loss falls from log V
towards log(genes of a type)."""
import argparse
import math
import os
import sys

import torch

sys.path.insert(0, os.path.join(os.path.dirname(os.path.abspath(__file__)), ".."))

import paper_2505_09326_amd as sph
from paper_2505_09326_amd.autograd import spherical_attention, token_embedding, vocab_cross_entropy


def cells(batch, length, genes, types, hidden_share, generator, device):
    """tokens, counts, targets [batch, length]: the hidden tokens are `genes`, targets are -100 where nothing is hidden."""
    per_type = genes // types
    kind = torch.randint(types, (batch, 1), generator=generator, device=device)
    own = kind * per_type + torch.randint(per_type, (batch, length), generator=generator, device=device)
    counts = torch.poisson(torch.full((batch, length), 2.0, device=device), generator=generator) + 1
    hidden = torch.rand((batch, length), generator=generator, device=device) < hidden_share
    return torch.where(hidden, genes, own), counts, torch.where(hidden, own, -100)


def train(steps=100, batch=8, length=512, genes=4000, types=20, heads=4, width=64, lr=3e-3, device="cuda:0", seed=0):
    """Losses and gradient norms of the steps."""
    g = torch.Generator(device=device).manual_seed(seed)
    D = heads * width
    new = lambda *shape, scale: (torch.randn(shape, generator=g, device=device) * scale).bfloat16().requires_grad_(True)
    table = new(genes + 1, D, scale=0.5 * D ** -0.5)           # the last row is the hidden token's
    Wq, Wk, Wv, Wo = (new(D, D, scale=D ** -0.5) for _ in range(4))
    weights = [table, Wq, Wk, Wv, Wo]
    masters = [w.detach().float() for w in weights]            # (the steps are smaller than bf16's)
    optimizer = torch.optim.Adam(masters, lr=lr)
    split = lambda x: x.view(batch, length, heads, width).transpose(1, 2).contiguous()
    losses, norms = [], []
    for _ in range(steps):
        tokens, counts, targets = cells(batch, length, genes, types, 0.15, g, device)
        X = token_embedding(tokens, table, torch.log1p(counts), math.sqrt(D))
        O = spherical_attention(split(X @ Wq), split(X @ Wk), split(X @ Wv))
        X = X + O.transpose(1, 2).reshape(batch, length, D) @ Wo
        loss = vocab_cross_entropy(X, table, targets)
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
    print(f"log V = {math.log(4001):.4f}, log(genes of a type) = {math.log(200):.4f}")

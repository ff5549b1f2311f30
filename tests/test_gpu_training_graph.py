"""A whole step, embedding, vocabulary loss, their gradients through autograd and clipping, captured into a graph: every replay gives what the entry points
called one by one give on the same inputs.  No eager autograd graph of the captured leaves exists before or beside the captured one."""
import pytest
import torch

import paper_2505_09326_amd as pkg
from paper_2505_09326_amd.autograd import token_embedding, vocab_cross_entropy

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("T,dtype", [(40, torch.float32), (300, torch.bfloat16), (2000, torch.float32)])
def test_a_captured_step(T, dtype):
    print("case captured step", T, dtype, flush=True)
    V, D = 700, 72
    g = torch.Generator(device=DEV).manual_seed(T)
    table, W = (torch.randn(V, D, generator=g, device=DEV).mul_(D ** -0.5).to(dtype).requires_grad_(True) for _ in range(2))
    tokens, mult = torch.randint(V, (T,), generator=g, device=DEV), torch.rand(T, generator=g, device=DEV)
    targets, one = torch.randint(-50, V, (T,), generator=g, device=DEV), torch.ones((), device=DEV)

    def by_hand():
        E, head = table.detach(), W.detach()
        X = pkg.sphattn_embed_fwd(tokens, E, mult, 3.0)
        _, lse, loss = pkg.sphattn_vocab_loss_fwd(X, head, targets, reduction="mean", all_rows=False)
        dX, dW = pkg.sphattn_vocab_loss_bwd(X, head, targets, lse, one, reduction="mean")
        grads = [pkg.sphattn_embed_bwd(tokens, dX, V, mult, 3.0), dW]
        return [loss, pkg.sphattn_clip_grads(grads, 0.01), *grads]

    def step():
        loss = vocab_cross_entropy(token_embedding(tokens, table, mult, 3.0), W, targets)
        grads = list(torch.autograd.grad(loss, (table, W), one))
        return [loss.detach(), pkg.sphattn_clip_grads(grads, 0.01), *grads]

    by_hand()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step()
    for turn in range(3):
        tokens.copy_(tokens.roll(turn + 1))
        targets.copy_(targets.flip(0))
        with torch.no_grad():
            W.mul_(0.9)
        for t in got:
            t.fill_(7.0)
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(got, by_hand()):
            assert torch.equal(a, b), turn

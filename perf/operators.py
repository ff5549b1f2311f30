"""The training-step operators around the attention, as they are timed: calls over the sizes that their users make them at.

  embed   sphattn_embed_fwd                 rows of a table of gene tokens, scaled, for inference
  lookup  autograd.token_embedding          the same in training: the rows and the gradient of the whole table
  score   sphattn_vocab_loss_fwd            -log softmax(X W^T)[target] of each row, for scoring
  loss    autograd.vocab_cross_entropy      the mean of that in training, with the gradients of X and W
  clip    sphattn_clip_grads                the 2-norm of all gradients together, and the gradients scaled down to a limit

Where `own` is false each is computed from elementary torch operations in fp32 and rounded once at the end.
"""
import math

import torch

own = False
DEV = "cuda"
_TORCH = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
_SIZE = {"f32": 4, "bf16": 2, "f16": 2}


def _embed(name, op, dtype, T, V, D, mult, tokens):
    return {"name": name, "op": op, "dtype": dtype, "T": T, "V": V, "D": D, "mult": mult, "tokens": tokens}


def _loss(name, op, dtype, T, V, D, share):
    return {"name": name, "op": op, "dtype": dtype, "T": T, "V": V, "D": D, "share": share}


def _clip(name, dtype, tensors, elements, max_norm):
    return {"name": name, "op": "clip", "dtype": dtype, "tensors": tensors, "elements": elements, "max_norm": max_norm}


def listed():
    return [
        # one token of one sequence: all latency
        _embed("embed_one_token", "embed", "bf16", 1, 32768, 1024, False, "zipf"),
        # two sequences of 8192 genes with their counts, 16 heads of 128
        _embed("embed_genes_16384", "embed", "bf16", 16384, 32768, 2048, True, "zipf"),
        # a training step's tokens: few common genes, many rare ones, most of a ragged table not there at all
        _embed("lookup_train_8192", "lookup", "bf16", 8192, 19999, 1024, True, "zipf"),
        # masked genes: half of the tokens are the one that stands for a hidden gene
        _embed("lookup_train_masked_32768", "lookup", "f32", 32768, 5003, 512, False, "masked"),
        # the log probability of one token after one row: reads W once
        _loss("score_one_row", "score", "bf16", 1, 32768, 1024, 1.0),
        # a scoring batch in half precision, every size odd, so that no row of W is aligned
        _loss("score_f16_odd", "score", "f16", 701, 20011, 515, 1.0),
        # a training step of an ordinary size: 8192 genes, 8 heads of 128
        _loss("loss_train_8192", "loss", "bf16", 8192, 32768, 1024, 1.0),
        # the largest: a wide model and a large vocabulary
        _loss("loss_train_large", "loss", "bf16", 8192, 65536, 2048, 1.0),
        # masked genes: only every seventh row or so has something to predict
        _loss("loss_train_masked_f16", "loss", "f16", 8000, 20011, 1024, 0.15),
        # fp32 training of a small model on one cell
        _loss("loss_train_f32", "loss", "f32", 1999, 8000, 512, 1.0),
        # a small model's gradients, which launches bound
        _clip("clip_small", "f32", 12, 400_000, 1.0),
        # the gradients of a model of some 200 million parameters, matrices and vectors
        _clip("clip_large", "bf16", 61, 200_000_000, 1.0),
    ]


# ---- drawn cases --------------------------------------------------------------------------------

_MOST_FLOPS = {"bf16": 5e12, "f16": 5e12, "f32": 6e11}


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng):
    D = _log_int(rng, 64, 2048)
    return D if rng.random() < 0.25 else max(64, D // 64 * 64)


def draw(rng):
    op = rng.choice(["embed", "lookup", "lookup", "score", "score", "loss", "loss", "loss", "clip", "clip"])
    dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
    if op in ("embed", "lookup"):
        case = _embed("", op, dtype, _log_int(rng, 1, 65536), _log_int(rng, 200, 65536), _width(rng),
                      rng.random() < 0.5, rng.choice(["zipf", "zipf", "masked", "even"]))
        while case["T"] * case["D"] > 1 << 25:
            case["T"] = int(case["T"] * 0.8)
    elif op in ("score", "loss"):
        case = _loss("", op, dtype, _log_int(rng, 1, 8192), _log_int(rng, 200, 65536), _width(rng),
                     rng.choice([1.0, 1.0, 0.9, 0.15]))
        while work(case)["flops"] > _MOST_FLOPS[dtype]:
            case["T"] = max(1, int(case["T"] * 0.8))
    else:
        tensors = _log_int(rng, 1, 61)
        case = _clip("", dtype, tensors, _log_int(rng, 100 * tensors, 100_000_000), rng.choice([0.5, 1.0, 1e6]))
    del case["name"]
    return case


# ---- inputs -------------------------------------------------------------------------------------

def _generator(case, seed):
    mix = 1000003 * (seed + 1) + 31 * case.get("T", 0) + 17 * case.get("V", 0) + case.get("D", case.get("elements", 0))
    return torch.Generator(device=DEV).manual_seed(mix)


def _randn(g, *shape):
    return torch.randn(shape, generator=g, device=DEV, dtype=torch.float32)


def _tokens(case, g):
    """Token ids [T] (int64): as often as genes occur, evenly, or half of them one and the same."""
    T, V = case["T"], case["V"]
    if case["tokens"] == "even":
        return torch.randint(V, (T,), generator=g, device=DEV)
    often = 1.0 / (10.0 + torch.arange(V, device=DEV, dtype=torch.float32))
    order = torch.randperm(V, generator=g, device=DEV)
    tokens = order[torch.multinomial(often, T, replacement=True, generator=g)]
    if case["tokens"] == "masked":
        hidden = torch.rand((T,), generator=g, device=DEV) < 0.5
        tokens = torch.where(hidden, torch.full_like(tokens, V - 1), tokens)
    return tokens


def _shapes(case):
    """A model's gradients: half of the tensors vectors, the rest matrices that share the elements."""
    n, total = case["tensors"], case["elements"]
    vectors = n // 2
    width = max(1, min(2048, total // (20 * n)))
    left = total - vectors * width
    matrices = n - vectors
    weights = [1 + i % 4 for i in range(matrices)]
    sizes = [max(1, left * w // sum(weights)) for w in weights]
    return [(width,)] * vectors + [((s // width, width) if s % width == 0 else (s,)) for s in sizes]


def _inputs(case, seed):
    g = _generator(case, seed)
    t16 = _TORCH[case["dtype"]]
    if case["op"] == "clip":
        shapes = _shapes(case)
        return {"grads": [(_randn(g, *s) * 10.0 ** ((i % 5) - 3)).to(t16) for i, s in enumerate(shapes)]}
    T, V, D = case["T"], case["V"], case["D"]
    if case["op"] in ("embed", "lookup"):
        t = {"tokens": _tokens(case, g), "table": _randn(g, V, D).mul_(D ** -0.5).to(t16), "scale": math.sqrt(D)}
        t["mult"] = torch.log1p(torch.poisson(torch.full((T,), 1.5, device=DEV), generator=g)) if case["mult"] else None
        if case["op"] == "lookup":
            t["dO"] = _randn(g, T, D).to(t16)
        return t
    # hidden states that already lean to their targets, as a model has them after some training
    W = _randn(g, V, D).mul_(2.0 * D ** -0.5).to(t16)
    targets = torch.randint(V, (T,), generator=g, device=DEV)
    X = (_randn(g, T, D) + W[targets].float() * torch.rand((T, 1), generator=g, device=DEV).mul_(2.0)).to(t16)
    if case["share"] < 1.0:
        rows = torch.randperm(T, generator=g, device=DEV)[_counted(case):]
        targets[rows] = -100
    return {"X": X, "W": W, "targets": targets}


def _counted(case):
    return max(1, round(case["share"] * case["T"]))


def _loss_scale(case):
    return 4096.0 if case["dtype"] == "f16" else 1.0


def prepare(case, seed):
    state = _inputs(case, seed)
    state["case"] = case
    if case["op"] == "clip":
        state["out"] = [torch.empty_like(x) for x in state["grads"]]
    if case["op"] == "lookup":
        state["table"].requires_grad_(True)
    if case["op"] == "loss":
        # half precision is trained with a scaled loss: small gradients would leave its range
        state["dloss"] = torch.tensor(_loss_scale(case), device=DEV)
        state["X"].requires_grad_(True)
        state["W"].requires_grad_(True)
    return state


# ---- one pass -----------------------------------------------------------------------------------

def run(state):
    return _run_own(state) if own else _run_plain(state)


def _run_own(state):
    import paper_2505_09326_amd as sph
    from paper_2505_09326_amd import autograd
    op = state["case"]["op"]
    if op == "embed":
        return sph.sphattn_embed_fwd(state["tokens"], state["table"], mult=state["mult"], scale=state["scale"])
    if op == "lookup":
        out = autograd.token_embedding(state["tokens"], state["table"], mult=state["mult"], scale=state["scale"])
        dtable, = torch.autograd.grad(out, (state["table"],), state["dO"])
        return [out.detach(), dtable]
    if op == "score":
        losses, lse = sph.sphattn_vocab_loss_fwd(state["X"], state["W"], state["targets"])
        return [losses, lse]
    if op == "loss":
        loss = autograd.vocab_cross_entropy(state["X"], state["W"], state["targets"])
        dX, dW = torch.autograd.grad(loss, (state["X"], state["W"]), state["dloss"])
        return [loss.detach(), dX, dW]
    norm = sph.sphattn_clip_grads(state["grads"], state["case"]["max_norm"], out=state["out"])
    return [norm, *state["out"]]


@torch.no_grad()
def _run_plain(state):
    case = state["case"]
    t16, op = _TORCH[case["dtype"]], case["op"]
    if op in ("embed", "lookup"):
        tokens, table = state["tokens"], state["table"]
        factor = state["scale"] if state["mult"] is None else (state["mult"] * state["scale"])[:, None]
        out = (table[tokens].float() * factor).to(t16)
        if op == "embed":
            return out
        dtable = torch.zeros(table.shape, dtype=torch.float32, device=DEV).index_add_(0, tokens, state["dO"].float() * factor)
        return [out, dtable.to(t16)]
    if op in ("score", "loss"):
        X, W, targets = state["X"].float(), state["W"].float(), state["targets"]
        counted = targets >= 0
        at = targets.clamp_min(0)[:, None]
        logits = X @ W.t()
        most = logits.amax(1, keepdim=True)
        lse = (logits - most).exp_().sum(1, keepdim=True).log_() + most
        losses = torch.where(counted, (lse - logits.gather(1, at))[:, 0], 0.0)
        if op == "score":
            return [losses, lse[:, 0]]
        n = counted.sum()
        dL = logits.sub_(lse).exp_()
        dL.scatter_add_(1, at, torch.full_like(lse, -1.0))
        dL.mul_((counted * state["dloss"] / n)[:, None])
        return [losses.sum() / n, (dL @ W).to(t16), (dL.t() @ X).to(t16)]
    grads = state["grads"]
    norm = torch.stack([x.float().square().sum() for x in grads]).sum().sqrt()
    factor = (case["max_norm"] / (norm + 1e-6)).clamp_max(1.0)
    torch._foreach_copy_(state["out"], [x.float() * factor for x in grads])
    return [norm, *state["out"]]


# ---- what a pass cannot do without --------------------------------------------------------------

def work(case):
    e = _SIZE[case["dtype"]]
    if case["op"] == "clip":
        n = sum(math.prod(s) for s in _shapes(case))
        return {"bytes": 2 * e * n, "flops": 3 * n}
    T, V, D = case["T"], case["V"], case["D"]
    if case["op"] in ("embed", "lookup"):
        # (of the table no more rows than there are tokens)
        nbytes = min(T, V) * D * e + T * D * e + 8 * T + (4 * T if case["mult"] else 0)
        if case["op"] == "lookup":
            nbytes += T * D * e + V * D * e
        return {"bytes": nbytes, "flops": T * D * (1 if case["op"] == "embed" else 3)}
    counted = _counted(case)
    nbytes = T * 8 + (T if case["op"] == "score" else counted) * D * e + V * D * e
    if case["op"] == "score":                      # (every row's log of the sum is asked for)
        return {"bytes": nbytes + 8 * T, "flops": 2 * T * D * V}
    return {"bytes": nbytes + T * D * e + V * D * e, "flops": 6 * counted * D * V}


# ---- the same in 64 bits ------------------------------------------------------------------------

def exact(case, seed):
    t = _inputs(case, seed)
    if case["op"] == "clip":
        squares = [float((x.double() ** 2).sum()) for x in t["grads"]]
        norm = math.sqrt(math.fsum(squares))
        factor = min(1.0, case["max_norm"] / (norm + 1e-6))
        return [torch.tensor(norm, dtype=torch.float64), *[x.double() * factor for x in t["grads"]]]
    T, V, D = case["T"], case["V"], case["D"]
    if case["op"] in ("embed", "lookup"):
        f = torch.full((T, 1), t["scale"], dtype=torch.float64, device=DEV)
        if t["mult"] is not None:
            f = f * t["mult"].double()[:, None]
        out = t["table"].double().index_select(0, t["tokens"]) * f
        if case["op"] == "embed":
            return out
        dtable = torch.zeros((V, D), dtype=torch.float64, device=DEV)
        dtable.index_add_(0, t["tokens"], t["dO"].double() * f)
        return [out, dtable]
    W, targets = t["W"].double(), t["targets"]
    Wt = W.t().contiguous()
    losses = torch.zeros(T, dtype=torch.float64, device=DEV)
    lses = torch.zeros_like(losses)
    n = int((targets >= 0).sum())
    dX = torch.zeros((T, D), dtype=torch.float64, device=DEV)
    dW = torch.zeros((V, D), dtype=torch.float64, device=DEV)
    step = max(1, (1 << 30) // (8 * V))            # 1 GB of logits at a time
    for i in range(0, T, step):
        x, y = t["X"][i:i + step].double(), targets[i:i + step]
        logits = x @ Wt
        lse = torch.logsumexp(logits, 1)
        lses[i:i + step] = lse
        rows = (y >= 0).nonzero()[:, 0]
        losses[i + rows] = lse[rows] - logits[rows, y[rows]]
        if case["op"] == "loss" and rows.numel():
            p = (logits[rows] - lse[rows, None]).exp()
            p[torch.arange(rows.numel(), device=DEV), y[rows]] -= 1.0
            p *= _loss_scale(case) / n
            dX[i + rows] = p @ W
            dW += p.t().contiguous() @ x[rows]
    if case["op"] == "score":
        return [losses, lses]
    return [losses.sum() / n, dX, dW]

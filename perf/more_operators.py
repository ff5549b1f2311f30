"""A layer's operators around the attention and training from a teacher, as they are timed: calls over the sizes that their users make them at.

  heads       sphattn_head_norm_rotary_fwd     queries and keys of a projection, normalised head by head, rotated by their positions and laid out
                                               for the attention; a single token's key goes into its place in a cache
  heads_train autograd.head_norm_rotary        the same in training, with the gradients of the projections and the norms' weights
  ffn         sphattn_gated_ffn_fwd            act(X Wg^T) * (X Wu^T), for inference
  ffn_train   autograd.gated_feed_forward      the same in training, with the gradients of X and both weights
  distill     sphattn_vocab_distill_fwd        the divergence of a student's vocabulary softmax from a teacher's top logits, for evaluation
  distill_train autograd.vocab_distillation    the mean of that in training, with the gradients of X and W

Where `own` is false each is computed from elementary torch operations in fp32 (angles in fp64) and rounded once at the end.
"""
import math

import torch

own = False
DEV = "cuda"
_TORCH = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
_SIZE = {"f32": 4, "bf16": 2, "f16": 2}
EPS = 1e-6


def _heads(name, op, dtype, B, N, Hq, Hk, d, axes, interleaved, far, cache=0):
    return {"name": name, "op": op, "dtype": dtype, "B": B, "N": N, "Hq": Hq, "Hk": Hk, "d": d, "axes": axes, "interleaved": interleaved,
            "far": far, "cache": cache}


def _ffn(name, op, dtype, T, D, F, act):
    return {"name": name, "op": op, "dtype": dtype, "T": T, "D": D, "F": F, "act": act}


def _distill(name, op, dtype, T, V, D, K, tau, share):
    return {"name": name, "op": op, "dtype": dtype, "T": T, "V": V, "D": D, "K": K, "tau": tau, "share": share}


def listed():
    return [
        # one new token of one sequence, far along, its key into a cache: all latency
        _heads("heads_one_token", "heads", "bf16", 1, 1, 16, 4, 128, 1, False, 30000, cache=4096),
        # two sequences of 8192, 16 heads of 128, queries and keys alike
        _heads("heads_prompts_16384", "heads", "bf16", 2, 8192, 16, 16, 128, 1, False, 0),
        # a training step of the same with keys shared by four heads
        _heads("heads_train_16384", "heads_train", "bf16", 2, 8192, 16, 4, 128, 1, False, 0),
        # fp32 training on patches of short films: three axes, neighbouring dimensions rotated, every count odd
        _heads("heads_train_axes_f32", "heads_train", "f32", 3, 2003, 9, 3, 64, 3, True, 100),
        # one row of a small model: reads the weights once
        _ffn("ffn_one_row", "ffn", "bf16", 1, 1024, 4096, "silu"),
        # a training step in half precision, every size odd, so that no row is aligned
        _ffn("ffn_train_f16_odd", "ffn_train", "f16", 1701, 515, 1371, "gelu"),
        # the largest: a training step of 8192 tokens of a wide model
        _ffn("ffn_train_large", "ffn_train", "bf16", 8192, 2048, 8192, "silu"),
        # fp32 training of a small model on one cell
        _ffn("ffn_train_f32", "ffn_train", "f32", 1999, 512, 2048, "silu"),
        # a few rows looked at between training steps: reads W once
        _distill("distill_few_rows", "distill", "bf16", 48, 32768, 1024, 64, 1.0, 1.0),
        # a training step of an ordinary size from a teacher's 64 best
        _distill("distill_train_8192", "distill_train", "bf16", 8192, 32768, 1024, 64, 1.0, 1.0),
        # masked genes: a third of the rows has a teacher's answer, some of them less than 20 of it; softened
        _distill("distill_train_masked_f16", "distill_train", "f16", 4001, 20011, 1024, 20, 2.0, 0.3),
        # fp32 training of a small model on one cell
        _distill("distill_train_f32", "distill_train", "f32", 1999, 8000, 512, 32, 1.5, 1.0),
    ]


# ---- drawn cases --------------------------------------------------------------------------------

_MOST_FLOPS = {"bf16": 1.6e12, "f16": 1.6e12, "f32": 2e11}


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng, lo, hi):
    n = _log_int(rng, lo, hi)
    return n if rng.random() < 0.25 else max(64, n // 64 * 64)


def draw(rng):
    op = rng.choice(["heads", "heads_train", "heads_train", "ffn", "ffn_train", "ffn_train", "distill", "distill_train", "distill_train"])
    dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
    if op in ("heads", "heads_train"):
        Hk = rng.choice([1, 2, 3, 4, 8, 16])
        case = _heads("", op, dtype, _log_int(rng, 1, 64), _log_int(rng, 1, 8192), Hk * rng.choice([1, 1, 2, 4]), Hk, rng.choice([64, 128]),
                      rng.choice([1, 1, 2, 3]), rng.random() < 0.4, rng.choice([0, 100, 30000, 1000000]))
        if op == "heads" and rng.random() < 0.4:
            case["N"] = 1
            case["cache"] = _log_int(rng, 16, 1024)
        while case["B"] * case["N"] * (case["Hq"] + case["Hk"]) * case["d"] > 1 << 26:
            case["B"], case["N"] = max(1, int(case["B"] * 0.8)), max(1, int(case["N"] * 0.8))
    elif op in ("ffn", "ffn_train"):
        case = _ffn("", op, dtype, _log_int(rng, 1, 8192), _width(rng, 64, 2048), _width(rng, 64, 8192), rng.choice(["silu", "silu", "gelu", "relu"]))
        while work(case)["flops"] > _MOST_FLOPS[dtype]:
            case["T"] = max(1, int(case["T"] * 0.8))
    else:
        case = _distill("", op, dtype, _log_int(rng, 1, 8192), _log_int(rng, 300, 50000), _width(rng, 64, 1024), _log_int(rng, 1, 128),
                        rng.choice([1.0, 1.0, 2.0, 4.0]), rng.choice([1.0, 1.0, 0.8, 0.2]))
        while work(case)["flops"] > _MOST_FLOPS[dtype]:
            case["T"] = max(1, int(case["T"] * 0.8))
    del case["name"]
    return case


# ---- inputs -------------------------------------------------------------------------------------

def _generator(case, seed):
    mix = 1000003 * (seed + 1) + 31 * case.get("T", case.get("N", 0)) + 17 * case.get("V", case.get("F", case.get("Hq", 0))) + case.get("D", case.get("d", 0))
    return torch.Generator(device=DEV).manual_seed(mix)


def _randn(g, *shape):
    return torch.randn(shape, generator=g, device=DEV, dtype=torch.float32)


def _rand(g, *shape):
    return torch.rand(shape, generator=g, device=DEV, dtype=torch.float32)


def _sections(case):
    """How many of the d/2 frequencies go by each axis."""
    half, axes = case["d"] // 2, case["axes"]
    rest = half // 4 if axes > 1 else half
    return [rest] + [(half - rest) // (axes - 1)] * (axes - 1) if axes > 1 else [half]


def _heads_inputs(case, g, t):
    B, N, Hq, Hk, d = (case[k] for k in ("B", "N", "Hq", "Hk", "d"))
    # one projection's output holds queries, keys and values side by side
    packed = (_randn(g, B, N, (Hq + 2 * Hk) * d) * (0.5 + _rand(g, B, N, 1))).to(t)
    s = {"packed": packed, "wq": (1.0 + 0.1 * _randn(g, d)).to(t), "wk": (1.0 + 0.1 * _randn(g, d)).to(t)}
    s["inv_freq"] = torch.pow(10000.0, -torch.arange(0, d, 2, device=DEV, dtype=torch.float64) / d).float()
    at = torch.arange(N, device=DEV)[None, :] + (torch.randint(case["far"], (B, 1), generator=g, device=DEV) if case["far"] else torch.zeros((B, 1), device=DEV, dtype=torch.int64))
    s["positions"] = at if case["axes"] == 1 else torch.stack([at // 64, at % 64 // 8, at % 8][:case["axes"]])
    if case["cache"]:
        s["cache"] = _randn(g, B, Hk, case["cache"], d).to(t)
        s["at"] = int(torch.randint(case["cache"], (1,), generator=g, device=DEV))
    if case["op"] == "heads_train":
        s["dQ"], s["dK"] = _randn(g, B, Hq, N, d).to(t), _randn(g, B, Hk, N, d).to(t)
    return s


def _ffn_inputs(case, g, t):
    T, D, F = case["T"], case["D"], case["F"]
    s = {"X": _randn(g, T, D).to(t), "Wg": (_randn(g, F, D) * (1.5 * D ** -0.5)).to(t), "Wu": (_randn(g, F, D) * D ** -0.5).to(t)}
    if case["op"] == "ffn_train":
        # (tokens' gradients are of different sizes)
        s["dH"] = (_randn(g, T, F) * torch.pow(10.0, -2.0 * _rand(g, T, 1))).to(t)
    return s


def _distill_inputs(case, g, t):
    T, V, D, K = case["T"], case["V"], case["D"], case["K"]
    W = (_randn(g, V, D) * (2.0 * D ** -0.5)).to(t)
    # K different ids a row, common ones more often than rare ones, and a teacher's logits for them, the best first
    often = torch.log(1.0 / (10.0 + torch.arange(V, device=DEV, dtype=torch.float32)))[torch.randperm(V, generator=g, device=DEV)]
    step = max(1, (1 << 28) // V)
    ids = torch.cat([(often - torch.log(-torch.log(_rand(g, min(step, T - i), V).clamp_(1e-7, 1.0 - 1e-6)))).topk(K, 1).indices for i in range(0, T, step)])
    teacher = (3.0 * _randn(g, T, K)).sort(1, descending=True).values.contiguous()
    X = _randn(g, T, D)
    for k in range(min(K, 4)):                     # hidden states that lean to the teacher's answers already
        X += W[ids[:, k]].float() * (_rand(g, T, 1) * 2.0 ** -k)
    if case["share"] < 1.0:
        ids[torch.arange(K, device=DEV)[None, :] >= torch.randint(1, 2 * K + 1, (T, 1), generator=g, device=DEV)] = -1
        ids[torch.randperm(T, generator=g, device=DEV)[_counted(case):]] = -1
    return {"X": X.to(t), "W": W, "ids": ids, "teacher": teacher}


def _counted(case):
    return max(1, round(case["share"] * case["T"]))


def _loss_scale(case):
    return 4096.0 if case["dtype"] == "f16" else 1.0


def _inputs(case, seed):
    g = _generator(case, seed)
    make = _heads_inputs if "Hq" in case else _ffn_inputs if "F" in case else _distill_inputs
    return make(case, g, _TORCH[case["dtype"]])


def _split(packed, case):
    """Queries [B,N,Hq,d] and keys [B,N,Hk,d], where the projection has left them."""
    B, N, Hq, Hk, d = (case[k] for k in ("B", "N", "Hq", "Hk", "d"))
    return packed[..., :Hq * d].view(B, N, Hq, d), packed[..., Hq * d:(Hq + Hk) * d].view(B, N, Hk, d)


def prepare(case, seed):
    state = _inputs(case, seed)
    state["case"] = case
    if "Hq" in case:
        state["q"], state["k"] = _split(state["packed"], case)
        state["sections"] = _sections(case)
        learned = ("q", "k", "wq", "wk")
    elif "F" in case:
        learned = ("X", "Wg", "Wu")
    else:
        # half precision is trained with a scaled loss: small gradients would leave its range
        state["dloss"] = torch.tensor(_loss_scale(case), device=DEV)
        learned = ("X", "W")
    if case["op"].endswith("_train"):
        for name in learned:
            state[name] = state[name].detach().requires_grad_(True)
    return state


# ---- one pass -----------------------------------------------------------------------------------

def run(state):
    return _run_own(state) if own else _run_plain(state)


def _run_own(state):
    import paper_2505_09326_amd as sph
    from paper_2505_09326_amd import autograd
    case = state["case"]
    op = case["op"]
    if op == "heads":
        K = state["cache"][:, :, state["at"]:state["at"] + 1] if case["cache"] else None
        Q, K = sph.sphattn_head_norm_rotary_fwd(state["q"], state["k"], state["wq"], state["wk"], positions=state["positions"], inv_freq=state["inv_freq"],
                                                sections=state["sections"], interleaved=case["interleaved"], eps=EPS, K=K)
        return [Q, state["cache"] if case["cache"] else K]
    if op == "heads_train":
        learned = (state["q"], state["k"], state["wq"], state["wk"])
        Q, K = autograd.head_norm_rotary(*learned, positions=state["positions"], inv_freq=state["inv_freq"], sections=state["sections"],
                                         interleaved=case["interleaved"], eps=EPS)
        grads = torch.autograd.grad((Q, K), learned, (state["dQ"], state["dK"]))
        return [Q.detach(), K.detach(), *grads]
    if op == "ffn":
        return sph.sphattn_gated_ffn_fwd(state["X"], state["Wg"], state["Wu"], activation=case["act"])
    if op == "ffn_train":
        learned = (state["X"], state["Wg"], state["Wu"])
        H = autograd.gated_feed_forward(*learned, activation=case["act"])
        return [H.detach(), *torch.autograd.grad(H, learned, state["dH"])]
    if op == "distill":
        losses, lse = sph.sphattn_vocab_distill_fwd(state["X"], state["W"], state["ids"], state["teacher"], temperature=case["tau"])
        return [losses, lse]
    loss = autograd.vocab_distillation(state["X"], state["W"], state["ids"], state["teacher"], temperature=case["tau"])
    dX, dW = torch.autograd.grad(loss, (state["X"], state["W"]), state["dloss"])
    return [loss.detach(), dX, dW]


@torch.no_grad()
def _run_plain(state):
    plain = _plain_heads if "Hq" in state["case"] else _plain_ffn if "F" in state["case"] else _plain_distill
    return plain(state, state["case"], _TORCH[state["case"]["dtype"]])


def _angles(state, case):
    """cos and sin [B,N,1,d/2]."""
    axis = torch.repeat_interleave(torch.arange(case["axes"], device=DEV), torch.tensor(state["sections"], device=DEV), output_size=case["d"] // 2)
    at = state["positions"][..., None].double() if case["axes"] == 1 else state["positions"][axis].permute(1, 2, 0).double()
    angle = at * state["inv_freq"].double()
    return angle.cos().float()[:, :, None], angle.sin().float()[:, :, None]


def _halves(x, interleaved):
    return (x[..., 0::2], x[..., 1::2]) if interleaved else x.chunk(2, -1)


def _whole(a, b, interleaved):
    return torch.stack((a, b), -1).flatten(-2) if interleaved else torch.cat((a, b), -1)


def _plain_heads(state, case, t):
    cos, sin = _angles(state, case)
    order, out, back = case["interleaved"], [], []
    for name in ("q", "k"):
        x, w = state[name].float(), state["w" + name].float()
        r = (x.square().mean(-1, keepdim=True) + EPS).rsqrt()
        n = x * r
        a, b = _halves(n * w, order)
        out.append(_whole(a * cos - b * sin, b * cos + a * sin, order).transpose(1, 2).contiguous().to(t))
        if case["op"] == "heads_train":
            a, b = _halves(state["d" + name.upper()].float().transpose(1, 2), order)
            dy = _whole(a * cos + b * sin, b * cos - a * sin, order)
            dn = dy * w
            back.append(((dn - n * (dn * n).mean(-1, keepdim=True)).mul_(r).to(t), (dy * n).sum((0, 1, 2)).to(t)))
    if case["cache"]:
        state["cache"][:, :, state["at"]] = out[1][:, :, 0]
        out[1] = state["cache"]
    if case["op"] == "heads_train":
        (dq, dwq), (dk, dwk) = back
        return [*out, dq, dk, dwq, dwk]
    return out


def _plain_ffn(state, case, t):
    X, Wg, Wu = (state[k].float() for k in ("X", "Wg", "Wu"))
    A, U = X @ Wg.t(), X @ Wu.t()
    if case["act"] == "relu":
        slope = (A > 0).float()
        act = A * slope
    else:
        gate = torch.sigmoid(A) if case["act"] == "silu" else 0.5 * (1.0 + torch.erf(A * math.sqrt(0.5)))
        act = A * gate
        slope = gate * (1.0 + A * (1.0 - gate)) if case["act"] == "silu" else gate + A * torch.exp(-0.5 * A * A) * (2.0 * math.pi) ** -0.5
    H = (act * U).to(t)
    if case["op"] == "ffn":
        return H
    dH = state["dH"].float()
    dA, dU = dH * U * slope, dH * act
    return [H, (dA @ Wg + dU @ Wu).to(t), (dA.t() @ X).to(t), (dU.t() @ X).to(t)]


def _plain_distill(state, case, t):
    X, W, ids, tau = state["X"].float(), state["W"].float(), state["ids"], case["tau"]
    there, at = ids >= 0, ids.clamp_min(0)
    counted = there.any(1)
    logits = (X @ W.t()).mul_(1.0 / tau)
    most = logits.amax(1, keepdim=True)
    lse = (logits - most).exp_().sum(1, keepdim=True).log_() + most
    best = torch.where(there, state["teacher"] / tau, -math.inf)
    best = best - torch.where(counted[:, None], best.amax(1, keepdim=True), 0.0)
    logp = best - best.exp().sum(1, keepdim=True).log()
    p = torch.where(there, logp.exp(), 0.0)
    terms = torch.where(there & (p > 0), p * (logp - logits.gather(1, at) + lse), 0.0)
    losses = tau * tau * terms.sum(1)
    lse = torch.where(counted[:, None], lse, 0.0)
    if case["op"] == "distill":
        return [losses, lse[:, 0]]
    n = counted.sum()
    dL = logits.sub_(lse).exp_()
    dL.scatter_add_(1, at, -p)
    dL.mul_((counted * state["dloss"] * tau / n)[:, None])
    return [losses.sum() / n, (dL @ W).to(t), (dL.t() @ X).to(t)]


# ---- what a pass cannot do without --------------------------------------------------------------

def work(case):
    e = _SIZE[case["dtype"]]
    train = case["op"].endswith("_train")
    if "Hq" in case:
        B, N, d, H = case["B"], case["N"], case["d"], case["Hq"] + case["Hk"]
        n = B * N * H * d
        nbytes = 2 * n * e + 2 * d * e + 2 * d + 8 * case["axes"] * B * N
        return {"bytes": nbytes + (2 * n * e + 2 * d * e if train else 0), "flops": n * (20 if train else 7)}
    if "F" in case:
        T, D, F = case["T"], case["D"], case["F"]
        once = (T * D + 2 * F * D) * e
        return {"bytes": once + T * F * e + (T * F * e + once if train else 0), "flops": (12 if train else 4) * T * F * D}
    T, V, D, K, counted = case["T"], case["V"], case["D"], case["K"], _counted(case)
    nbytes = 12 * T * K + counted * D * e + V * D * e
    if not train:
        return {"bytes": nbytes + 8 * T, "flops": 2 * counted * D * V}
    return {"bytes": nbytes + T * D * e + V * D * e, "flops": 6 * counted * D * V}


# ---- the same in 64 bits ------------------------------------------------------------------------

def exact(case, seed):
    return (_exact_heads if "Hq" in case else _exact_ffn if "F" in case else _exact_distill)(case, _inputs(case, seed))


def _exact_heads(case, s):
    B, N, d, half = case["B"], case["N"], case["d"], case["d"] // 2
    turn = torch.empty((B, N, 1, half), dtype=torch.float64, device=DEV)
    first = 0
    for axis, n in enumerate(_sections(case)):
        at = (s["positions"] if case["axes"] == 1 else s["positions"][axis]).double()
        turn[:, :, 0, first:first + n] = at[..., None] * s["inv_freq"][first:first + n].double()
        first += n
    turn = torch.polar(torch.ones_like(turn), turn)

    def paired(x):                                 # the two dimensions that turn together as a complex number
        x = x.unflatten(-1, (half, 2) if case["interleaved"] else (2, half))
        return torch.complex(x[..., 0], x[..., 1]) if case["interleaved"] else torch.complex(x[..., 0, :], x[..., 1, :])

    def apart(z):
        return torch.stack((z.real, z.imag), -1 if case["interleaved"] else -2).flatten(-2)

    outs, grads, weights = [], [], []
    for x, w, dO in zip(_split(s["packed"], case), (s["wq"], s["wk"]), (s.get("dQ"), s.get("dK"))):
        x, w = x.double(), w.double()
        norm = (x.pow(2).sum(-1, keepdim=True) / d + EPS).sqrt()
        unit = x / norm
        outs.append(apart(paired(unit * w) * turn).permute(0, 2, 1, 3).contiguous())
        if dO is not None:
            dy = apart(paired(dO.double().permute(0, 2, 1, 3)) * turn.conj())
            weights.append((dy * unit).sum(dim=(0, 1, 2)))
            along = (dy * w * unit).sum(-1, keepdim=True) / d
            grads.append((dy * w - along * unit) / norm)
    if case["cache"]:
        cache = s["cache"].double()
        cache[:, :, s["at"]:s["at"] + 1] = outs[1]
        outs[1] = cache
    return [*outs, *grads, *weights]


def _exact_ffn(case, s):
    X, Wg, Wu = (s[k].double() for k in ("X", "Wg", "Wu"))
    A, U = X @ Wg.t().contiguous(), X @ Wu.t().contiguous()
    if case["act"] == "silu":
        e = torch.exp(-A)
        act, slope = A / (1.0 + e), (1.0 + e + A * e) / (1.0 + e) ** 2
    elif case["act"] == "gelu":
        below = torch.special.erfc(-A / math.sqrt(2.0)) / 2.0
        act, slope = A * below, below + A * torch.exp(-A * A / 2.0) / math.sqrt(2.0 * math.pi)
    else:
        act, slope = A.clamp_min(0.0), torch.where(A > 0, 1.0, 0.0).double()
    H = act * U
    if case["op"] == "ffn":
        return H
    dH = s["dH"].double()
    dA, dU = dH * U * slope, dH * act
    return [H, dA @ Wg + dU @ Wu, dA.t().contiguous() @ X, dU.t().contiguous() @ X]


def _exact_distill(case, s):
    T, V, D, K, tau = case["T"], case["V"], case["D"], case["K"], case["tau"]
    W, ids = s["W"].double(), s["ids"]
    Wt = W.t().contiguous()
    losses, lses = torch.zeros(T, dtype=torch.float64, device=DEV), torch.zeros(T, dtype=torch.float64, device=DEV)
    dX, dW = torch.zeros((T, D), dtype=torch.float64, device=DEV), torch.zeros((V, D), dtype=torch.float64, device=DEV)
    rows = (ids >= 0).any(1).nonzero()[:, 0]
    n = rows.numel()
    step = max(1, (1 << 30) // (8 * V))            # 1 GB of logits at a time
    for i in range(0, n, step):
        r = rows[i:i + step]
        x, y = s["X"][r].double(), ids[r]
        there = y >= 0
        p = torch.softmax(torch.where(there, s["teacher"][r].double() / tau, -math.inf), 1)
        logits = (x @ Wt) / tau
        lse = torch.logsumexp(logits, 1)
        student = logits.gather(1, y.clamp_min(0)) - lse[:, None]
        lses[r] = lse
        losses[r] = tau ** 2 * (torch.special.xlogy(p, p) - torch.where(there, p * student, 0.0)).sum(1)
        if case["op"] == "distill_train":
            G = (logits - lse[:, None]).exp()
            G.scatter_add_(1, y.clamp_min(0), -p)
            G *= tau * _loss_scale(case) / n
            dX[r] = G @ W
            dW += G.t().contiguous() @ x
    if case["op"] == "distill":
        return [losses, lses]
    return [losses.sum() / n, dX, dW]

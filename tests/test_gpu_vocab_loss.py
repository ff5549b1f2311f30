"""Cross entropy over a vocabulary and its gradients against the formulas in 64 bits.

Tolerances, from the roundings (u = 2^-24; e = eps / 2 of the storage type):
  logits   sums of D products in fp32: off by at most a = u (D + 4) A with A = |scale| max_t sum_k |x_k| max_v |w_vk|, in fp32 storage
           2^-21 A more for the products of parts that are left out
  lse      a, and the sum over V of exponentials each a few u off, joined in 64ths and tiles: a + u (V / 64 + 100) + 8 u |lse|
  loss     a difference of two such: 2 a + ...
  G        g (p (lse's tolerance + a) + 4 u) from the exponential and the subtraction, rounded to the type: e |G|; in fp16 never below
           2^-39 of the largest g
  dX, dW   the sum of those times |w| (|x|), u n of the sum of magnitudes for adding n terms, e of the result"""
import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U = 2.0 ** -24
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


@pytest.fixture(scope="module")
def pkg():
    import paper_2505_09326_amd as p
    p.load_library()
    return p


def _inputs(T, V, D, dtype, seed, share=0.8, ids=torch.int64, offset=0, spread=2.0):
    g = torch.Generator(device=DEV).manual_seed(seed)
    t = TYPES[dtype]

    def make(rows, factor):
        x = torch.randn(rows * D, generator=g, device=DEV) * factor
        return torch.empty(rows * D + offset, dtype=t, device=DEV)[offset:].copy_(x.to(t)).view(rows, D)
    X, W = make(T, 1.0), make(V, spread * D ** -0.5)
    targets = torch.randint(V, (T,), generator=g, device=DEV)
    targets[torch.rand(T, generator=g, device=DEV) >= share] = -100
    return X, W, targets.to(ids)


class Exact:
    """Losses, gradients and how far each may be off."""

    def __init__(self, X, W, targets, scale, dloss, reduction):
        x, w, t = X.double(), W.double(), X.dtype
        T, V, D = x.shape[0], w.shape[0], x.shape[1]
        e = torch.finfo(t).eps / 2
        wt = w.t().contiguous()
        logits = (x @ wt) * scale
        A = abs(scale) * float((x.abs() @ wt.abs().amax(1)).max()) if T else 0.0
        a = U * (D + 4) * A + (2.0 ** -21 * A if t == torch.float32 else 0.0)
        self.lse = torch.logsumexp(logits, 1)
        self.lse_tol = a + U * (V / 64 + 100) + 8 * U * self.lse.abs()
        self.counted = targets >= 0
        at = targets.long().clamp_min(0)[:, None]
        mine = logits.gather(1, at)[:, 0]
        self.losses = torch.where(self.counted, self.lse - mine, 0.0)
        self.loss_tol = torch.where(self.counted, self.lse_tol + a + 8 * U * mine.abs(), 0.0)
        n = max(1, int(self.counted.sum()))
        g = dloss.double() if reduction == "none" else dloss.double().expand(T) / (n if reduction == "mean" else 1)
        g = torch.where(self.counted, g, 0.0)[:, None]
        p = (logits - self.lse[:, None]).exp()
        G = p.clone()
        G.scatter_add_(1, at, torch.full((T, 1), -1.0, dtype=torch.float64, device=DEV))
        G *= g * scale
        off = (p * (self.lse_tol[:, None] + a) + 4 * U) * (g * scale).abs() + e * G.abs()
        if t == torch.float16 and T:
            off += 2.0 ** -38 * float((g * scale).abs().max()) * (g != 0)
        size = G.abs()
        tiny = torch.finfo(t).tiny * torch.finfo(t).eps
        extra = 2.0 ** -21 if t == torch.float32 else 0.0
        self.dX, self.dW = G @ w, G.t().contiguous() @ x
        self.dX_tol = off @ w.abs() + (U * (V + 4) + extra) * (size @ w.abs()) + e * self.dX.abs() + tiny
        sw, sx = size.t().contiguous() @ x.abs(), off.t().contiguous() @ x.abs()
        self.dW_tol = sx + (U * (T + 4) + extra) * sw + e * self.dW.abs() + tiny


def _near(got, want, tol, what):
    far = (got.double() - want).abs() - tol
    assert not bool(got.isnan().any()), what
    assert far.numel() == 0 or float(far.max()) <= 0, (what, float(far.max()))


SHAPES = [  # T, V, D, dtype, share of rows that count, scale, ids, offset
    (1, 1, 1, "f32", 1.0, 1.0, torch.int64, 0),
    (1, 1000, 64, "bf16", 1.0, 1.0, torch.int64, 0),
    (3, 5, 7, "f16", 0.7, 1.0, torch.int32, 0),
    (16, 129, 40, "bf16", 0.8, 0.5, torch.int64, 0),
    (17, 2000, 72, "bf16", 0.8, 1.0, torch.int32, 0),
    (64, 257, 515, "f16", 0.8, 1.0, torch.int64, 0),
    (65, 3000, 33, "bf16", 0.8, 1.0, torch.int64, 0),
    (130, 255, 128, "f16", 0.8, -0.25, torch.int64, 0),
    (300, 1111, 200, "bf16", 0.5, 1.0, torch.int64, 5),
    (513, 4097, 96, "f32", 0.8, 1.0, torch.int64, 0),
    (300, 700, 130, "f32", 0.3, 2.0, torch.int64, 1),
    (40, 3001, 64, "f32", 0.9, 1.0, torch.int64, 0),
    (7, 600, 48, "f32", 1.0, 1.0, torch.int64, 0),
    (4096, 300, 64, "bf16", 0.15, 1.0, torch.int64, 0),
    (2048, 12000, 256, "bf16", 1.0, 1.0, torch.int64, 0),          # tiles of 256 x 256
    (2500, 10000, 320, "f16", 0.9, 1.0, torch.int64, 0),
    (1999, 8000, 136, "f32", 1.0, 1.0, torch.int64, 0),
    (4096, 33000, 64, "bf16", 0.5, 1.0, torch.int64, 0),           # two pieces of the vocabulary
    (1500, 30000, 40, "f32", 1.0, 1.0, torch.int64, 0),            # two pieces, three parts
]


@pytest.mark.parametrize("T,V,D,dtype,share,scale,ids,offset", SHAPES)
def test_losses_and_gradients(pkg, T, V, D, dtype, share, scale, ids, offset):
    X, W, targets = _inputs(T, V, D, dtype, 5 + T + V + D, share, ids, offset)
    dloss = torch.tensor(3.0 if dtype != "f16" else 512.0, device=DEV)
    want = Exact(X, W, targets, scale, dloss, "mean")
    losses, lse = pkg.sphattn_vocab_loss_fwd(X, W, targets, scale)
    _near(lse, want.lse, want.lse_tol, "lse")
    _near(losses, want.losses, want.loss_tol, "losses")
    losses, lse, mean = pkg.sphattn_vocab_loss_fwd(X, W, targets, scale, "mean", all_rows=False)
    counted = want.counted
    _near(losses, want.losses, want.loss_tol, "losses of the rows that count")
    _near(lse, torch.where(counted, want.lse, 0.0), want.lse_tol, "their lse")
    n = max(1, int(counted.sum()))
    _near(mean, want.losses.sum() / n, want.loss_tol.sum() / n + 2 * U * want.losses.sum() / n, "mean")
    dX, dW = pkg.sphattn_vocab_loss_bwd(X, W, targets, lse, dloss, scale, "mean")
    _near(dX, want.dX, want.dX_tol, "dX")
    _near(dW, want.dW, want.dW_tol, "dW")
    assert bool((dX[~counted] == 0).all())
    again = pkg.sphattn_vocab_loss_bwd(X, W, targets, lse, dloss, scale, "mean")
    assert torch.equal(dX, again[0]) and torch.equal(dW, again[1])


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
def test_gradients_row_by_row(pkg, dtype):
    """One gradient per row, over twelve powers of ten, and one gradient at a time."""
    X, W, targets = _inputs(200, 777, 72, dtype, 3)
    g = torch.Generator(device=DEV).manual_seed(8)
    dloss = torch.randn(200, generator=g, device=DEV) * 10.0 ** torch.randint(-2, 2, (200,), generator=g, device=DEV)
    dloss[targets < 0] = 1e30                      # of rows that do not count: not to be looked at
    want = Exact(X, W, targets, 1.0, torch.where(targets < 0, 0.0, dloss), "none")
    _, lse = pkg.sphattn_vocab_loss_fwd(X, W, targets)
    dX, dW = pkg.sphattn_vocab_loss_bwd(X, W, targets, lse, dloss)
    _near(dX, want.dX, want.dX_tol, "dX")
    _near(dW, want.dW, want.dW_tol, "dW")
    assert torch.equal(pkg.sphattn_vocab_loss_bwd(X, W, targets, lse, dloss, want_dW=False)[0], dX)
    assert torch.equal(pkg.sphattn_vocab_loss_bwd(X, W, targets, lse, dloss, want_dX=False)[1], dW)
    want = Exact(X, W, targets, 1.0, torch.tensor(-2.0, device=DEV), "sum")
    dX, dW = pkg.sphattn_vocab_loss_bwd(X, W, targets, lse, torch.tensor(-2.0, device=DEV), reduction="sum")
    _near(dX, want.dX, want.dX_tol, "dX of the sum")
    _near(dW, want.dW, want.dW_tol, "dW of the sum")


def test_small_gradients_of_half_precision(pkg):
    """A mean over many rows makes gradients far below fp16's normal numbers: they are lost in the results at most, not before."""
    X, W, targets = _inputs(1000, 500, 64, "f16", 9, 1.0)
    _, lse = pkg.sphattn_vocab_loss_fwd(X, W, targets)
    small = pkg.sphattn_vocab_loss_bwd(X, W, targets, lse, torch.tensor(2.0 ** -4, device=DEV), reduction="mean")
    large = pkg.sphattn_vocab_loss_bwd(X, W, targets, lse, torch.tensor(2.0 ** 10, device=DEV), reduction="mean")
    for s, l in zip(small, large):                 # the same sums, scaled by a power of two
        assert bool(((s.double() - l.double() * 2.0 ** -14).abs() <= 2.0 ** -11 * s.double().abs() + 2.0 ** -25).all())


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
def test_no_row_counts(pkg, dtype):
    X, W, targets = _inputs(70, 300, 40, dtype, 4, 0.0)
    for reduction in ("sum", "mean"):
        losses, lse, total = pkg.sphattn_vocab_loss_fwd(X, W, targets, reduction=reduction, all_rows=False)
        assert float(total) == 0 and bool((losses == 0).all()) and bool((lse == 0).all())
        dX, dW = pkg.sphattn_vocab_loss_bwd(X, W, targets, lse, torch.ones((), device=DEV), reduction=reduction,
                                            dX=torch.full_like(X, 3.0), dW=torch.full_like(W, 3.0))
        assert bool((dX == 0).all()) and bool((dW == 0).all())


def test_no_rows(pkg):
    W = torch.randn(300, 40, device=DEV)
    X, targets = torch.empty(0, 40, device=DEV), torch.empty(0, dtype=torch.int64, device=DEV)
    losses, lse, mean = pkg.sphattn_vocab_loss_fwd(X, W, targets, reduction="mean")
    assert losses.shape == lse.shape == (0,) and float(mean) == 0
    dX, dW = pkg.sphattn_vocab_loss_bwd(X, W, targets, lse, torch.ones((), device=DEV), reduction="mean", dW=torch.full_like(W, 3.0))
    assert dX.shape == (0, 40) and bool((dW == 0).all())


def test_target_outside_the_vocabulary(pkg):
    X, W, targets = _inputs(50, 300, 40, "bf16", 4, 1.0)
    targets[7], targets[8] = 300, 2 ** 40
    losses, lse = pkg.sphattn_vocab_loss_fwd(X, W, targets)
    bad = torch.zeros(50, dtype=torch.bool, device=DEV)
    bad[7:9] = True
    assert torch.equal(losses.isnan(), bad) and torch.equal(lse.isnan(), bad)
    dX, dW = pkg.sphattn_vocab_loss_bwd(X, W, targets, lse, torch.ones(50, device=DEV))
    assert torch.equal(dX.isnan().all(1), bad) and torch.equal(dX.isnan().any(1), bad) and bool(dW.isnan().all())


def test_infinite_logits(pkg):
    X, W, targets = _inputs(40, 500, 64, "bf16", 4, 1.0)
    X[:, 0] = X[:, 0].abs() + 1
    targets[:] = 11
    W[13] = 0
    W[13, 0] = -1e30                               # far below all others: no weight, no gradient
    losses, lse = pkg.sphattn_vocab_loss_fwd(X, W, targets)
    want = Exact(X, torch.cat([W[:13], W[14:]]), targets, 1.0, torch.ones(40, device=DEV), "none")
    assert bool(((lse.double() - want.lse).abs() <= want.lse_tol).all())
    dX, dW = pkg.sphattn_vocab_loss_bwd(X, W, targets, lse, torch.ones(40, device=DEV))
    assert bool(dX.isfinite().all()) and bool((dW[13] == 0).all())
    W[13, 0] = float("-inf")                       # a logit of -inf (its zeros meet finite values only)
    assert torch.equal(pkg.sphattn_vocab_loss_fwd(X, W, targets)[1], lse)
    W[13, 0] = float("inf")
    losses, lse = pkg.sphattn_vocab_loss_fwd(X, W, targets)
    assert bool((lse == float("inf")).all()) and bool((losses == float("inf")).all())
    W[13, 0] = 0
    X[5, 3] = float("nan")                         # one row's own
    losses, lse = pkg.sphattn_vocab_loss_fwd(X, W, targets)
    assert int(losses.isnan().sum()) == 1 and bool(losses[5].isnan())


@pytest.mark.parametrize("shift", [-300.0, 300.0])
def test_logits_far_from_zero(pkg, shift):
    """No exponential of a logit itself is ever formed."""
    X, W, targets = _inputs(70, 400, 32, "f32", 6, 1.0)
    X[:, 0], W[:, 0] = shift, 1.0
    want = Exact(X, W, targets, 1.0, torch.ones(70, device=DEV), "none")
    losses, lse = pkg.sphattn_vocab_loss_fwd(X, W, targets)
    _near(lse, want.lse, want.lse_tol, "lse")
    _near(losses, want.losses, want.loss_tol, "losses")


def test_autograd_against_differences(pkg):
    from paper_2505_09326_amd.autograd import vocab_cross_entropy
    X, W, targets = _inputs(60, 300, 48, "f32", 12, 0.8)
    X.requires_grad_(True)
    W.requires_grad_(True)
    loss = vocab_cross_entropy(X.view(3, 20, 48), W, targets.view(3, 20), scale=0.7)
    dX, dW = torch.autograd.grad(loss, (X, W))
    g = torch.Generator(device=DEV).manual_seed(2)
    stepX, stepW = torch.randn(60, 48, generator=g, device=DEV), torch.randn(300, 48, generator=g, device=DEV)

    def at(h):
        x, w = X.detach().double() + h * stepX.double(), W.detach().double() + h * stepW.double()
        logits = 0.7 * (x @ w.t().contiguous())
        rows = (targets >= 0).nonzero()[:, 0]
        return float((torch.logsumexp(logits, 1)[rows] - logits[rows, targets[rows]]).mean())
    h = 1e-4
    slope = (at(h) - at(-h)) / (2 * h)
    got = float((dX.double() * stepX.double()).sum() + (dW.double() * stepW.double()).sum())
    size = float((dX.abs() * stepX.abs()).sum() + (dW.abs() * stepW.abs()).sum())
    assert got == pytest.approx(slope, abs=1e-6 * size + 1e-6)     # (differences: h^2 times a third derivative of order 1)
    per_row = vocab_cross_entropy(X.view(3, 20, 48), W, targets.view(3, 20), 0.7, "none")
    assert per_row.shape == (3, 20)
    frozen, = torch.autograd.grad(vocab_cross_entropy(X, W.detach(), targets, 0.7), (X,))
    assert torch.equal(frozen, dX)


def test_other_stream_and_graph(pkg):
    X, W, targets = _inputs(300, 2000, 128, "bf16", 31, 0.7)
    one = torch.ones((), device=DEV)

    def step():
        losses, lse, mean = pkg.sphattn_vocab_loss_fwd(X, W, targets, reduction="mean", all_rows=False)
        return (mean, *pkg.sphattn_vocab_loss_bwd(X, W, targets, lse, one, reduction="mean"))
    want = step()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = step()
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step()
    for turn in range(3):
        for t in got:
            t.fill_(7.0)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want)), turn
        targets.copy_(targets.roll(turn + 1))      # other rows count in the next replay
        want = step()

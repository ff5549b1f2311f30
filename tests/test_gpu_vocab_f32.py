"""Cross entropy over a vocabulary in fp32 where the split into parts could go wrong: tensors far from 1, elements far below their tensor's
largest, rows that do not count with any content, more than one piece of the vocabulary.

Tolerances: X and W are split into two fp16 parts each (2^-22 of an element, or 2^-39 of the tensor's largest), the product of the second parts is
left out (2^-22): a term is off by 3 2^-22, a sum of n by n u more (u = 2^-24)."""
import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U, TERM = 2.0 ** -24, 3 * 2.0 ** -22


@pytest.fixture(scope="module")
def pkg():
    import paper_2505_09326_amd as p
    p.load_library()
    yield p
    # what the 64-bit products left in the allocator (a library's workspace inside a large segment) is no memory of later tests
    torch._C._cuda_clearCublasWorkspaces()
    torch.cuda.empty_cache()


def _exact(X, W, targets, scale):
    """lse, losses, and dX and dW of the losses' sum, in 64 bits, each with what it may be off by."""
    x, w = X.double(), W.double()
    x = torch.where(targets[:, None] >= 0, x, 0.0)
    wt = w.t().contiguous()
    logits = scale * (x @ wt)
    floor = 2.0 ** -39 * abs(scale) * (float(x.abs().max()) * wt.abs().sum(0)[None] + float(w.abs().max()) * x.abs().sum(1)[:, None])
    a = (TERM + (X.shape[1] + 4) * U) * abs(scale) * (x.abs() @ wt.abs()) + floor
    lse = torch.logsumexp(logits, 1)
    lse_tol = a.amax(1) + U * (W.shape[0] / 64 + 100) + 8 * U * lse.abs()
    at = targets.clamp_min(0)[:, None]
    losses = lse - logits.gather(1, at)[:, 0]
    counted = targets >= 0
    p = (logits - lse[:, None]).exp()
    off = p * (a + lse_tol[:, None]) + 8 * U
    p.scatter_add_(1, at, torch.full_like(p[:, :1], -1.0))
    G, off = (t * counted[:, None] * abs(scale) for t in (p, off))
    off = off + TERM * G.abs() + 2.0 ** -38 * abs(scale)
    dX, dW = G * (1 if scale > 0 else -1) @ w, (G * (1 if scale > 0 else -1)).t().contiguous() @ x
    dX_tol = off @ w.abs() + (W.shape[0] + 4) * U * (G.abs() @ w.abs()) + 2.0 ** -39 * float(w.abs().max()) * G.abs().sum(1)[:, None]
    dW_tol = off.t().contiguous() @ x.abs() + (X.shape[0] + 4) * U * (G.abs().t().contiguous() @ x.abs()) + 2.0 ** -39 * float(x.abs().max()) * G.abs().sum(0)[:, None]
    return counted, (lse, lse_tol), (losses, lse_tol + a.amax(1) + 8 * U * losses.abs()), (dX, dX_tol + U * dX.abs()), (dW, dW_tol + U * dW.abs())


def _check(pkg, X, W, targets, scale):
    counted, lse, losses, dX, dW = _exact(X, W, targets, scale)
    got_losses, got_lse, total = pkg.sphattn_vocab_loss_fwd(X, W, targets, scale, "sum", all_rows=False)
    gX, gW = pkg.sphattn_vocab_loss_bwd(X, W, targets, got_lse, torch.ones((), device=DEV), scale, "sum")
    for name, got, (want, tol) in (("lse", got_lse[counted], [t[counted] for t in lse]), ("losses", got_losses[counted], [t[counted] for t in losses]),
                                   ("dX", gX, dX), ("dW", gW, dW)):
        assert bool(got.isfinite().all()), name
        far = (got.double() - want).abs() - tol
        assert float(far.max()) <= 0, (name, float(far.max()))
    assert bool((gX[~counted] == 0).all()) and bool((got_losses[~counted] == 0).all())


def _inputs(T, V, D, seed, share=0.8):
    g = torch.Generator(device=DEV).manual_seed(seed)
    X, W = torch.randn(T, D, generator=g, device=DEV), torch.randn(V, D, generator=g, device=DEV) * 2 * D ** -0.5
    targets = torch.randint(V, (T,), generator=g, device=DEV)
    targets[torch.rand(T, generator=g, device=DEV) >= share] = -1
    targets[0] = 0
    return X, W, targets, g


@pytest.mark.parametrize("T,V,D", [(5, 300, 40), (70, 1000, 72), (1100, 2000, 33)])
@pytest.mark.parametrize("x,w", [(1e20, 1e-20), (1e-25, 1e25), (2.0 ** 100, 2.0 ** -100)])
def test_tensors_far_from_one(pkg, T, V, D, x, w):
    X, W, targets, _ = _inputs(T, V, D, 1)
    _check(pkg, X * x, W * w, targets, 1.0)
    _check(pkg, X * 1e3, W * 1e3, targets, -1e-6)


def test_elements_far_below_the_largest(pkg):
    X, W, targets, g = _inputs(200, 700, 64, 2)
    W *= 10.0 ** -torch.randint(0, 12, (700, 1), generator=g, device=DEV).float()
    X *= 10.0 ** -torch.randint(0, 12, (200, 1), generator=g, device=DEV).float()
    X[3], W[5] = 0, 0
    _check(pkg, X, W, targets, 1.0)


@pytest.mark.parametrize("T", [30, 300, 1500])
@pytest.mark.parametrize("fill", [float("nan"), float("inf"), 3e38])
def test_rows_that_do_not_count_may_hold_anything(pkg, T, fill):
    X, W, targets, _ = _inputs(T, 500, 48, 3, 0.5)
    want = pkg.sphattn_vocab_loss_fwd(X, W, targets, reduction="mean", all_rows=False)
    grads = pkg.sphattn_vocab_loss_bwd(X, W, targets, want[1], torch.ones((), device=DEV), reduction="mean")
    X[targets < 0] = fill
    assert all(torch.equal(a, b) for a, b in zip(pkg.sphattn_vocab_loss_fwd(X, W, targets, reduction="mean", all_rows=False), want))
    assert all(torch.equal(a, b) for a, b in zip(pkg.sphattn_vocab_loss_bwd(X, W, targets, want[1], torch.ones((), device=DEV), reduction="mean"), grads))


def test_zeros(pkg):
    X, W, targets, _ = _inputs(20, 100, 16, 4)
    for x, w in ((torch.zeros_like(X), W), (X, torch.zeros_like(W)), (torch.zeros_like(X), torch.zeros_like(W))):
        _check(pkg, x, w, targets, 1.0)


def test_two_pieces_of_the_vocabulary(pkg):
    X, W, targets, _ = _inputs(4096, 20000, 40, 5)
    _check(pkg, X, W, targets, 1.0)


@pytest.mark.parametrize("T,V,D,offset", [(1, 1, 1, 0), (2, 63, 3, 0), (16, 130, 20, 0), (17, 5000, 100, 0), (40, 777, 64, 1), (64, 1000, 257, 0), (64, 129, 66, 2), (33, 300_001, 5, 0)])
def test_few_rows(pkg, T, V, D, offset):
    """Up to 64 rows are multiplied as fp32; 300001 ids are two pieces."""
    X, W, targets, _ = _inputs(T, V, D, 6)
    moved = lambda t: torch.empty(t.numel() + offset, device=DEV)[offset:].copy_(t.reshape(-1)).view(t.shape)
    _check(pkg, moved(X), moved(W), targets, 0.5)
    targets[1:] = -1
    _check(pkg, moved(X), moved(W), targets, -1.0)

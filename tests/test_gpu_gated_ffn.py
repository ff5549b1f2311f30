"""The gated feed-forward product and its gradients against the formulas in 64 bits.

Tolerances (u = 2^-24, e = eps / 2 of the storage type):
  A, U     a = (D + 4) u sum_k |x_k w_k|; fp32 with parts (more than 64 rows, and the gradients): 3 2^-22 more of each term, and elements to 2^-51 of their row's largest
  act      its slope (1.13 at most) times A's, and 12 u of |A| (in 16 bits and gelu 2e-7 |A|: a formula of 1.5e-7); its slope: 1.2 (silu: 0.5) times A's, and 2 u (16 + |A|) (gelu 6e-7)
  H        the product's, e |H|
  dA, dB   the product's and the rounding to the storage type, e (fp32: 2^-24); fp16: 2^-24 of a value that the largest of the row (of all rows for dW) brings to 2^13 or
           more, so 2^-37 of what the norms allow for it
  dX, dW   the sum of those of its terms, (n + 4) u of the terms' sizes for adding n of them (fp32: 2^-21 more for products of parts left out), e of the result."""
import math

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


def _inputs(T, D, F, dtype, seed, spread=1.5):
    g = torch.Generator(device=DEV).manual_seed(seed)
    r = lambda *s: torch.randn(s, generator=g, device=DEV)
    t = TYPES[dtype]
    # (tokens' gradients of different sizes)
    return r(T, D).to(t), (r(F, D) * spread * D ** -0.5).to(t), (r(F, D) * D ** -0.5).to(t), (r(T, F) * torch.pow(10.0, -3.0 * torch.rand((T, 1), generator=g, device=DEV))).to(t)


def _gate(A, act):
    if act == "relu":
        return A.clamp_min(0.0), (A > 0).double()
    if act == "silu":
        s = torch.sigmoid(A)
        return A * s, s * (1 + A * torch.sigmoid(-A))
    below = 0.5 * torch.special.erfc(-A * math.sqrt(0.5))
    return A * below, below + A * torch.exp(-0.5 * A * A) / math.sqrt(2 * math.pi)


def _projections(X, W, parts):
    x, w = X.double(), W.double()
    wt = w.t().contiguous()
    size = x.abs() @ wt.abs()
    tol = (X.shape[1] + 4) * U * size
    if parts:
        tol += 3 * 2.0 ** -22 * size + 2.0 ** -50 * (x.abs().amax(1)[:, None] * wt.abs().sum(0)[None] + wt.abs().amax(0)[None] * x.abs().sum(1)[:, None])
    return x @ wt, tol


def _exact(X, Wg, Wu, act, dH=None, parts=False):
    """(H, tolerance), or with dH the gradients with theirs, both without the result's own rounding."""
    t = X.dtype
    e = torch.finfo(t).eps / 2
    (A, ta), (B, tb) = _projections(X, Wg, parts), _projections(X, Wu, parts)
    value, slope = _gate(A, act)
    near = 0.0
    if act == "relu":                                          # where A may be of the other sign the slope is any
        near = (A.abs() <= ta).double()
    gelu16 = act == "gelu" and t != torch.float32
    tv = 1.13 * ta + A.abs() * (2e-7 if gelu16 else 12 * U)
    ts = {"silu": 0.51, "gelu": 0.81, "relu": 0.0}[act] * ta + (6e-7 if gelu16 else 2 * U * (16 + A.abs())) + near
    if dH is None:
        return value * B, tv * B.abs() + value.abs() * tb + tv * tb + 2 * U * (value * B).abs()
    d = dH.double()
    dA, dB = d * B * slope, d * value
    tA = d.abs() * (slope.abs() * tb + B.abs() * ts + ts * tb) + 3 * U * dA.abs()
    tB = d.abs() * tv + 2 * U * dB.abs()
    round_to = e if t != torch.float32 else U
    tA, tB = tA + round_to * (dA.abs() + tA), tB + round_to * (dB.abs() + tB)
    row = every = 0.0
    if t == torch.float16:
        w = max(float(W.double().norm(dim=1).max()) for W in (Wg, Wu))
        row = (X.double().norm(dim=1) * d.abs().amax(1) * w * 1.13 * 2.0 ** -37)[:, None]
        every = row.max()
    x, wg, wu = X.double(), Wg.double(), Wu.double()
    more = 2.0 ** -21 if t == torch.float32 else 0.0
    T, F = d.shape
    dX, sX = dA @ wg + dB @ wu, dA.abs() @ wg.abs() + dB.abs() @ wu.abs()
    tX = (tA + row) @ wg.abs() + (tB + row) @ wu.abs() + ((2 * F + 40) * U + more) * sX
    out = [(dX, tX)]
    for m, tol in ((dA, tA), (dB, tB)):
        mt = m.t().contiguous()
        out.append((mt @ x, (tol + every).t().contiguous() @ x.abs() + ((T + 40) * U + more) * (mt.abs() @ x.abs())))
    return out


def _near(got, want, tol, what):
    fi = torch.finfo(got.dtype)
    past = want.to(got.dtype).isinf()                          # what the type holds as infinite: 65520 and more in fp16
    got, want = torch.where(past & (got == want.to(got.dtype)), 0.0, got.double()), torch.where(past, 0.0, want)
    off = (got - want).abs()
    allowed = tol * (1 + fi.eps) + fi.eps / 2 * want.abs() * (1 + 2.0 ** -10) + fi.tiny * fi.eps
    bad = ~(off <= allowed)
    assert not bad.any(), f"{what}: {int(bad.sum())} of {bad.numel()}, worst {float((off / allowed.clamp_min(1e-300)).max()):.2f} of its tolerance"


CASES = [  # T, D, F
    (1, 64, 64), (1, 1024, 4096), (1, 515, 1371), (2, 1, 1), (16, 128, 17), (17, 96, 130), (32, 2048, 100), (33, 72, 255), (64, 40, 300),
    (33, 8192, 2048), (64, 2050, 8191),                        # (few rows of large weights: in tiles in 16 bits)
    (65, 64, 64), (129, 200, 65), (300, 515, 333), (257, 1000, 1200), (1000, 256, 96), (2500, 64, 136), (700, 2048, 640), (2048, 512, 1024)]


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("T,D,F", CASES)
def test_against_the_formulas(pkg, T, D, F, dtype):
    act = ["silu", "gelu", "relu"][(T + D + F) % 3]
    X, Wg, Wu, dH = _inputs(T, D, F, dtype, T + 3 * D + 5 * F)
    H = pkg.sphattn_gated_ffn_fwd(X, Wg, Wu, act)
    _near(H, *_exact(X, Wg, Wu, act, parts=dtype == "f32"), "H")
    grads = pkg.sphattn_gated_ffn_bwd(X, Wg, Wu, dH, act)
    for name, got, (want, tol) in zip(("dX", "dWg", "dWu"), grads, _exact(X, Wg, Wu, act, dH, parts=dtype == "f32")):
        _near(got, want, tol, name)
    assert torch.equal(H, pkg.sphattn_gated_ffn_fwd(X, Wg, Wu, act))
    for a, b in zip(grads, pkg.sphattn_gated_ffn_bwd(X, Wg, Wu, dH, act)):
        assert torch.equal(a, b)


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("act", ["silu", "gelu", "relu"])
@pytest.mark.parametrize("T", [5, 100])
def test_activations_over_their_range(pkg, T, act, dtype):
    """A from far below to far above 0, each value as one product, and what is not finite."""
    t = TYPES[dtype]
    values = torch.cat([torch.linspace(-30, 30, 601), torch.tensor([0.0, -0.0, 1e-4, -1e-4, 60.0, -60.0, 90.0, -90.0, 3e4, -3e4])]).to(DEV).to(t)
    F = values.numel()
    X = torch.zeros(T, 8, device=DEV, dtype=t)
    X[:, 0] = 1
    Wg, Wu = torch.zeros(F, 8, device=DEV, dtype=t), torch.zeros(F, 8, device=DEV, dtype=t)
    Wg[:, 0], Wu[:, 0] = values, 1
    H = pkg.sphattn_gated_ffn_fwd(X, Wg, Wu, act)
    value, slope = _gate(values.double(), act)
    tol = values.double().abs() * (2e-7 if act == "gelu" and dtype != "f32" else 12 * U) + U * value.abs()
    if dtype == "f32" or act != "gelu":                        # the tails too, each to its own size, down to where fp32's exponential ends
        own = value.abs() * (4 * values.double().abs() ** 2 + 24) * U + 1e-33
        tol = torch.minimum(tol, own)
    _near(H, value.expand(T, F), tol.expand(T, F), "H")
    dH = torch.ones(T, F, device=DEV, dtype=t)
    got = pkg.sphattn_gated_ffn_bwd(X, Wg, Wu, dH, act)
    want = _exact(X, Wg, Wu, act, dH, parts=dtype == "f32")
    for name, g, (w, tl) in zip(("dX", "dWg", "dWu"), got, want):
        _near(g, w, tl, name)
    nan = X.clone()
    nan[T - 1, 0] = float("nan")
    again = pkg.sphattn_gated_ffn_fwd(nan, Wg, Wu, act)
    assert torch.equal(again[:T - 1], H[:T - 1]) and again[T - 1].isnan().all()


@pytest.mark.parametrize("T", [3, 90])
def test_infinite_rows_of_fp32_are_the_formula(pkg, T):
    X, Wg, Wu, _ = _inputs(T, 72, 200, "f32", 1)
    Wg[7, 3], Wg[11, 5], Wu[12, 70] = float("-inf"), float("inf"), float("inf")
    X[1, 4] = float("inf")
    got = pkg.sphattn_gated_ffn_fwd(X, Wg, Wu, "relu").double()
    A, B = X.double() @ Wg.double().t(), X.double() @ Wu.double().t()
    want = torch.where(A <= 0, 0.0, A) * B
    fine = want.isfinite()
    assert torch.equal(fine, got.isfinite()) and torch.equal(want.isnan(), got.isnan()) and torch.equal(want[want.isinf()], got[got.isinf()])
    assert (got - want)[fine].abs().max() < 1e-3
    assert fine.sum() > 100 * T and not fine[1].any()


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("T,D,F", [(3, 64, 100), (200, 129, 257)])
def test_any_alignment_and_nothing_behind_the_ends(pkg, T, D, F, dtype):
    X, Wg, Wu, dH = _inputs(T, D, F, dtype, 2)
    want = pkg.sphattn_gated_ffn_fwd(X, Wg, Wu), *pkg.sphattn_gated_ffn_bwd(X, Wg, Wu, dH)

    def shifted(t, fill=None):
        flat = torch.full((t.numel() + 40,), 7.0, device=DEV, dtype=t.dtype)
        if fill is None:
            flat[3:3 + t.numel()] = t.flatten()
        return flat, flat[3:3 + t.numel()].view(t.shape)
    x, wg, wu, d = (shifted(t)[1] for t in (X, Wg, Wu, dH))
    outs = [shifted(t, 7.0) for t in want]
    pkg.sphattn_gated_ffn_fwd(x, wg, wu, H=outs[0][1])
    pkg.sphattn_gated_ffn_bwd(x, wg, wu, d, dX=outs[1][1], dWg=outs[2][1], dWu=outs[3][1])
    for (flat, view), w in zip(outs, want):
        assert torch.equal(view, w) and (flat[:3] == 7).all() and (flat[3 + w.numel():] == 7).all()


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
def test_one_gradient_at_a_time(pkg, dtype):
    X, Wg, Wu, dH = _inputs(150, 80, 120, dtype, 4)
    full = pkg.sphattn_gated_ffn_bwd(X, Wg, Wu, dH)
    for i in range(3):
        wants = {n: j == i for j, n in enumerate(("want_dX", "want_dWg", "want_dWu"))}
        only = pkg.sphattn_gated_ffn_bwd(X, Wg, Wu, dH, **wants)
        assert [t is not None for t in only] == [j == i for j in range(3)] and torch.equal(only[i], full[i])


def test_no_rows(pkg):
    for dtype in TYPES:
        _, Wg, Wu, _ = _inputs(1, 40, 50, dtype, 5)
        X = torch.empty(0, 40, device=DEV, dtype=TYPES[dtype])
        H = pkg.sphattn_gated_ffn_fwd(X, Wg, Wu)
        assert H.shape == (0, 50)
        dX, dWg, dWu = pkg.sphattn_gated_ffn_bwd(X, Wg, Wu, H)
        assert dX.shape == X.shape and (dWg == 0).all() and (dWu == 0).all()
        only = pkg.sphattn_gated_ffn_bwd(X, Wg, Wu, H, want_dWg=False, want_dWu=False)
        assert only[0].shape == X.shape and only[1] is only[2] is None


@pytest.mark.parametrize("scale", [2.0 ** -13, 1.0, 512.0])
def test_fp16_gradients_of_any_size(pkg, scale):
    """Row by row and column by column each to its own size: dA and dB would leave the type's range without their factors."""
    T, D, F = 130, 256, 300
    X, Wg, Wu, dH = _inputs(T, D, F, "f16", 6)
    X, dH = (X.float() * 4).half(), (dH.float() * scale).half()
    Wu = (Wu.float() * 8).half()
    for name, g, (w, tol) in zip(("dX", "dWg", "dWu"), pkg.sphattn_gated_ffn_bwd(X, Wg, Wu, dH), _exact(X, Wg, Wu, "silu", dH)):
        if w.abs().max() < 6e4:
            _near(g, w, tol, name)


def test_autograd(pkg):
    from paper_2505_09326_amd import autograd
    X, Wg, Wu, dH = _inputs(60, 48, 72, "bf16", 8)
    leaves = [t.clone().requires_grad_(True) for t in (X.view(4, 15, 48), Wg, Wu)]
    H = autograd.gated_feed_forward(*leaves, activation="gelu")
    assert H.shape == (4, 15, 72)
    grads = torch.autograd.grad(H, leaves, dH.view(4, 15, 72))
    for a, b in zip(grads, pkg.sphattn_gated_ffn_bwd(X, Wg, Wu, dH, "gelu")):
        assert torch.equal(a.reshape(b.shape), b)
    only, = torch.autograd.grad(autograd.gated_feed_forward(X, Wg, leaves[2]).sum(), (leaves[2],))
    assert torch.equal(only, pkg.sphattn_gated_ffn_bwd(X, Wg, Wu, torch.ones_like(dH), want_dX=False, want_dWg=False)[2])
    shared = Wg.clone().requires_grad_(True)                   # one weight in both places, rows of no token
    g, = torch.autograd.grad(autograd.gated_feed_forward(X[None, :0], shared, shared).sum(), (shared,))
    assert (g == 0).all()
    with pytest.raises(RuntimeError):
        first, = torch.autograd.grad(autograd.gated_feed_forward(*leaves).sum(), leaves[:1], create_graph=True)
        first.sum().backward()
    with pytest.raises(TypeError):
        autograd.gated_feed_forward(X, Wg.float(), Wu)


def test_gradients_against_differences(pkg):
    """Central differences of the formula in 64 bits along random directions, in fp32 (a step of 2^-9 of the norm 1: third derivatives below 2^-14 of the
    largest gradient)."""
    T, D, F = 70, 40, 56
    X, Wg, Wu, dH = _inputs(T, D, F, "f32", 9)
    grads = pkg.sphattn_gated_ffn_bwd(X, Wg, Wu, dH, "silu")
    at = [t.double() for t in (X, Wg, Wu)]
    g = torch.Generator(device=DEV).manual_seed(3)

    def value(x, a, b):
        return float((_gate(x @ a.t().contiguous(), "silu")[0] * (x @ b.t().contiguous()) * dH.double()).sum())
    for i in range(3):
        step = torch.randn(at[i].shape, generator=g, device=DEV, dtype=torch.float64)
        step *= 2.0 ** -9 / step.norm()
        up, down = (value(*[t + s * step if j == i else t for j, t in enumerate(at)]) for s in (1, -1))
        assert abs((up - down) / 2 - float((grads[i].double() * step).sum())) <= 2.0 ** -14 * float(grads[i].norm()) * 2.0 ** -9


@pytest.mark.parametrize("dtype,T", [("bf16", 4), ("bf16", 300), ("f16", 300), ("f32", 300)])
def test_graph_replays(pkg, dtype, T):
    X, Wg, Wu, dH = _inputs(T, 128, 384, dtype, 10)
    call = lambda: (pkg.sphattn_gated_ffn_fwd(X, Wg, Wu), *pkg.sphattn_gated_ffn_bwd(X, Wg, Wu, dH))
    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = call()
    for i in range(3):
        X.mul_(1.03125)
        dH.add_(0.125)
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(out, call()):
            assert torch.equal(a, b), i


def test_more_values_than_32_bits_count(pkg):
    """H and dH of 2^32 elements and more: their last rows are those of a call of their own."""
    T, D, F = 33000, 64, 131072
    g = torch.Generator(device=DEV).manual_seed(31)
    X = torch.randn(T, D, generator=g, device=DEV).bfloat16()
    Wg, Wu = (torch.randn(F, D, generator=g, device=DEV).mul_(D ** -0.5).bfloat16() for _ in range(2))
    few = slice(T - 80, T)
    H = pkg.sphattn_gated_ffn_fwd(X, Wg, Wu)
    assert torch.equal(H[few], pkg.sphattn_gated_ffn_fwd(X[few], Wg, Wu))
    dH = H                                                     # (any values will do; zeros but for the last rows)
    dH[:T - 80].zero_()
    dX, dWg, dWu = pkg.sphattn_gated_ffn_bwd(X, Wg, Wu, dH)
    want = pkg.sphattn_gated_ffn_bwd(X[few], Wg, Wu, dH[few].contiguous())
    assert (dX[:T - 80] == 0).all()
    for got, w in zip((dX[few], dWg, dWu), want):              # (the order of the sums is another: fp32's rounding, and a step of bf16 where that decides)
        off = (got.double() - w.double()).abs()
        assert (off <= 2.0 ** -7 * w.double().abs() + (2 * F + 40) * U * float(w.abs().max())).all()


@pytest.mark.parametrize("T,D,F", [(249, 320, 6144), (1649, 71, 1024), (3000, 64, 1300)])
def test_relu_beside_zero(pkg, T, D, F):
    """Of so many values of A some are so near 0 that sums in fp32 put them on the other side; one such slope is 1 / sqrt(T F / 2), 4e-4 and more, of dX.  With all slopes
    right the gradients are off by some 2^-21 of their terms: 2^-17 of their norms is far from either."""
    X, Wg, Wu, dH = _inputs(T, D, F, "f32", 249)
    near = X.double() @ Wg.double().t().contiguous()
    sides = int(((near > 0) != (X @ Wg.t() > 0)).sum())        # (how many a library's product has there: for the reader)
    grads = pkg.sphattn_gated_ffn_bwd(X, Wg, Wu, dH, "relu")
    for name, got, (want, _) in zip(("dX", "dWg", "dWu"), grads, _exact(X, Wg, Wu, "relu", dH, parts=True)):
        assert float((got.double() - want).norm() / want.norm()) < 2.0 ** -17, (name, sides)

"""Gates far from 0, masks of the type's lowest value and infinite ones, against the formulas in 64 bits.

A is one product and exact but for fp32's two parts (more than 64 rows, and the gradients), 2^-22 of it.  Tolerances (u = 2^-24, e = eps / 2 of the storage type, f = 8 u + 2^-22):
  act     above 0 f |a|; below -100 the formula has less than 1e-41, and from -87 to -104 an exponential below 2^-126 is 0, 104 times that
  slope   beyond 100 it is 0 or 1 to f; nearer ones f (1 + |a|)
Nothing in these grows with a gate below 0."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U = 2.0 ** -24
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
FAR = {"f32": [100.0, 104.0, 120.0, 1e3, 3e4, 1e5, 1e10, 1e19, 1e20, 1e30, 1e36, 1e38, 3e38], "bf16": [100.0, 104.0, 120.0, 1e3, 1e10, 1e19, 1e20, 1e30, 1e38, 3e38],
       "f16": [100.0, 104.0, 120.0, 1e3, 6e4]}


@pytest.fixture(scope="module")
def pkg():
    import paper_2505_09326_amd as p
    p.load_library()
    return p


def _gate(A, act):
    if act == "relu":
        return A.clamp_min(0.0), (A > 0).double()
    if act == "silu":
        s = torch.sigmoid(A)
        return A * s, s * (1 + A * torch.sigmoid(-A))
    below = 0.5 * torch.special.erfc(-A * math.sqrt(0.5))
    return A * below, below + A * torch.exp(-0.5 * A * A) / math.sqrt(2 * math.pi)


def _one_product(values, T, dtype):
    """X, Wg and Wu with A[t, f] = values[f] and U = 1."""
    t = TYPES[dtype]
    F = values.numel()
    X, Wg, Wu = torch.zeros(T, 8, device=DEV, dtype=t), torch.zeros(F, 8, device=DEV, dtype=t), torch.zeros(F, 8, device=DEV, dtype=t)
    X[:, 0], Wg[:, 0], Wu[:, 0] = 1, values, 1
    return X, Wg, Wu


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("act", ["silu", "gelu", "relu"])
@pytest.mark.parametrize("T", [1, 5, 40, 100, 1000])
def test_far_gates(pkg, T, act, dtype):
    t, e = TYPES[dtype], torch.finfo(TYPES[dtype]).eps / 2
    f = 8 * U + 2.0 ** -22
    far = torch.tensor(FAR[dtype], dtype=torch.float64)
    values = torch.cat([far, -far, torch.tensor([torch.finfo(t).min, torch.finfo(t).max, -60.0, -87.0, -88.0, -90.0, -95.0, 88.0, 0.0])]).to(DEV).to(t)
    v = values.double()
    value, slope = _gate(v, act)
    X, Wg, Wu = _one_product(values, T, dtype)
    H = pkg.sphattn_gated_ffn_fwd(X, Wg, Wu, act)
    tol = torch.where(v > 0, f * v, 104 * 2.0 ** -126 + 1e-4 * value.abs()) + torch.finfo(t).tiny * torch.finfo(t).eps
    for row in (0, T - 1):
        off = (H[row].double() - value).abs()
        assert (off <= tol + e * value.abs() * (1 + 2.0 ** -10)).all(), (row, values[off > tol + e * value.abs()], H[row])
    # dA = dH slope and dB = dH act, seen in the weights' gradients of one row that has a gradient
    dH = torch.zeros(T, values.numel(), device=DEV, dtype=t)
    dH[T // 2] = 0.5
    dX, dWg, dWu = pkg.sphattn_gated_ffn_bwd(X, Wg, Wu, dH, act)
    near = torch.where(v.abs() < 100, 1 + v.abs(), 1.0)
    assert ((dWg[:, 0].double() - 0.5 * slope).abs() <= f * near + 2 * e * slope.abs() + (2.0 ** -22 if dtype == "f16" else 0.0)).all(), (values, dWg[:, 0])
    # (fp16: dA and dB are kept to 2^-37 of what the norms allow, 0.5 times 6.5e4 times 1.13: 2^-22)
    assert ((dWu[:, 0].double() - 0.5 * value).abs() <= tol + 2 * e * value.abs() + (2.0 ** -22 if dtype == "f16" else 0.0)).all(), (values, dWu[:, 0])


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("act", ["silu", "gelu", "relu"])
@pytest.mark.parametrize("T", [3, 200])
def test_masked_gates_leave_nothing(pkg, T, act, dtype):
    """Gates that a bias of the type's lowest value masks: outputs and gradients of 0, however large the weights that the gradients are multiplied with."""
    t = TYPES[dtype]
    X, Wg, Wu = _one_product(torch.full((72,), torch.finfo(t).min, device=DEV), T, dtype)
    dH = torch.ones(T, 72, device=DEV, dtype=t)
    assert (pkg.sphattn_gated_ffn_fwd(X, Wg, Wu, act) == 0).all()
    for g in pkg.sphattn_gated_ffn_bwd(X, Wg, Wu, dH, act):
        assert (g == 0).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("act", ["silu", "gelu", "relu"])
@pytest.mark.parametrize("T", [3, 40, 90])
def test_infinite_rows_are_the_formula(pkg, T, act, dtype):
    """Infinite elements of X and of either weight: infinite and NaN results where the formula has them, the others untouched."""
    g = torch.Generator(device=DEV).manual_seed(T)
    X, Wg, Wu = (torch.randn(s, 72, generator=g, device=DEV).to(TYPES[dtype]) for s in (T, 200, 200))
    clean = pkg.sphattn_gated_ffn_fwd(X, Wg, Wu, act)
    Wg[7, 3], Wg[11, 5], Wu[12, 70] = float("-inf"), float("inf"), float("inf")
    X[1, 4] = float("inf")
    got = pkg.sphattn_gated_ffn_fwd(X, Wg, Wu, act).double()
    A, B = X.double() @ Wg.double().t().contiguous(), X.double() @ Wu.double().t().contiguous()
    value = _gate(A, act)[0] if act != "relu" else torch.where(A <= 0, 0.0, A)
    # (act is held in fp32: gelu at -16 is 1e-57, which is 0 there, and times an infinite U no number instead of an infinite one; among the numbers that fp32 has
    # fewer bits for, 2^-152 to 2^-120, it may be either)
    want = torch.where(value.abs() < 2.0 ** -126, 0.0, value) * B
    either = B.isinf() & (value.abs() > 2.0 ** -152) & (value.abs() < 2.0 ** -120)
    want, got = want.masked_fill(either, 0.0), got.masked_fill(either, 0.0)
    assert either.sum() < 8
    fine = want.isfinite()
    assert torch.equal(fine, got.isfinite()) and torch.equal(want.isnan(), got.isnan()) and torch.equal(want[want.isinf()], got[got.isinf()])
    rows = torch.ones(T, 200, dtype=torch.bool, device=DEV)
    rows[1], rows[:, [7, 11, 12]] = False, False
    assert fine[rows].all()
    size = X.double().nan_to_num(posinf=0).abs() @ Wg.double().nan_to_num(posinf=0, neginf=0).abs().t().contiguous()
    other = X.double().nan_to_num(posinf=0).abs() @ Wu.double().nan_to_num(posinf=0, neginf=0).abs().t().contiguous()
    # (either way of forming the sums is off by (72 + 4) u and 3 2^-22 of their terms at most, act's slope by 1.13 of that)
    tol = 2 * (76 * U + 3 * 2.0 ** -22) * 1.13 * size * other * 2 + torch.finfo(TYPES[dtype]).eps * clean.double().abs()
    assert ((got - clean.double()).abs() <= tol)[rows].all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("act", ["silu", "gelu", "relu"])
@pytest.mark.parametrize("T", [3, 200, 4200])
def test_closed_gates_beside_large_gradients(pkg, T, act, dtype):
    """dH U of 1e40 where the slope is 0: 0, and where it is 1 but dH 0 too."""
    t = TYPES[dtype]
    X, Wg, Wu = _one_product(torch.full((72,), -1000.0, device=DEV), T, dtype)
    Wg[5], Wu[:, 0] = 1000.0, 1e20
    dH = torch.full((T, 72), 1e20, device=DEV, dtype=t)
    dH[:, 5] = 0
    for g in pkg.sphattn_gated_ffn_bwd(X, Wg, Wu, dH, act):
        assert (g == 0).all()

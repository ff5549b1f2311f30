"""fp16 gradients of units far below the others: each row of dWg and dWu to its own size.

Tolerances are those of test_gpu_gated_ffn.py but for what the type has for small numbers: dA's column f is brought to 2^13 .. 2^14 of what its largest |dH| |x| and its own |w| allow
(the norms' product, 1.13 for act's slope), so half of its smallest step, 2^-25, is 2^-37 of that."""
import pytest
import torch

from test_gpu_gated_ffn import U, _gate, _inputs, _near, _projections

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.fixture(scope="module")
def pkg():
    import paper_2505_09326_amd as p
    p.load_library()
    return p


def _units(X, Wg, Wu, dH, act):
    """(dWg, tolerance), (dWu, tolerance) in 64 bits."""
    e = torch.finfo(torch.float16).eps / 2
    (A, ta), (B, tb) = _projections(X, Wg, False), _projections(X, Wu, False)
    value, slope = _gate(A, act)
    assert act == "silu"
    tv, ts = 1.13 * ta + 12 * U * A.abs(), 0.51 * ta + 2 * U * (16 + A.abs())
    d, x = dH.double(), X.double()
    out = []
    top = (d.abs() * x.norm(dim=1)[:, None]).amax(0)
    for m, t, w in ((d * B * slope, d.abs() * (slope.abs() * tb + B.abs() * ts + ts * tb), Wu), (d * value, d.abs() * tv, Wg)):
        t = t + 3 * U * m.abs()
        t = t + e * (m.abs() + t) + 2.0 ** -37 * 1.13 * top * w.double().norm(dim=1)
        mt, tt = m.t().contiguous(), t.t().contiguous()
        out.append((mt @ x, tt @ x.abs() + (X.shape[0] + 40) * U * (mt.abs() @ x.abs())))
    return out


@pytest.mark.parametrize("T,D,F", [(300, 256, 600), (1000, 256, 1400), (700, 131, 515), (5000, 64, 96), (9000, 40, 1030), (2100, 512, 2048)])
def test_small_units(pkg, T, D, F):
    X, Wg, Wu, _ = _inputs(T, D, F, "f16", T + F)
    g = torch.Generator(device=DEV).manual_seed(F)
    X = (X.float() / 16).half()
    Wg, Wu = (Wg.float() * 16).half(), (Wu.float() * 2.0 ** 12).half()                        # A of 1.5, U of 2^8
    dH = torch.randn(T, F, generator=g, device=DEV) * 2
    small = torch.arange(F, device=DEV) % 7 == 3
    dH[:, small] *= 2.0 ** -11
    Wu[small] = (Wu[small].float() * 2.0 ** -12).half()
    dH = dH.half()
    _, dWg, dWu = pkg.sphattn_gated_ffn_bwd(X, Wg, Wu, dH, "silu")
    for name, got, (want, tol) in zip(("dWg", "dWu"), (dWg, dWu), _units(X, Wg, Wu, dH, "silu")):
        assert want.abs().max() < 6e4
        _near(got, want, tol, name)
        # (bounds for a sum's every term grow with their number, what they make of it with its root: each unit as a whole is off by its terms' roundings and its own, e / sqrt(3) of
        # them in the mean each, e together)
        off = (got.double() - want)[small].norm(dim=1) / want[small].norm(dim=1)
        assert off.max() < 2 * torch.finfo(torch.float16).eps / 2, (name, off.max())


def test_rows_of_very_different_size(pkg):
    """Tokens whose X is a thousand times the others' but that have no gradient take no bits from the rest, nor does one of infinite gradients in other columns."""
    T, D, F = 500, 128, 300
    X, Wg, Wu, dH = _inputs(T, D, F, "f16", 3)
    X = (X.float() / 64).half()
    X[7] *= 4096
    dH[7] = 0
    dH = (dH.float() * 2.0 ** -6).half()
    got = pkg.sphattn_gated_ffn_bwd(X, Wg, Wu, dH, "silu")
    for g, (want, tol) in zip(got[1:], _units(X, Wg, Wu, dH, "silu")):
        _near(g, want, tol, "units")
    dH[9, 5] = float("inf")
    again = pkg.sphattn_gated_ffn_bwd(X, Wg, Wu, dH, "silu")
    others = torch.arange(F, device=DEV) != 5
    for a, b in zip(again[1:], got[1:]):
        assert torch.equal(a[others], b[others]) and not a[5].isfinite().any()
    assert not again[0][9].isfinite().any()
    rows = torch.arange(T, device=DEV) != 9
    assert torch.equal(again[0][rows], got[0][rows])


def test_no_gradient_at_all(pkg):
    X, Wg, Wu, dH = _inputs(400, 64, 700, "f16", 4)
    for t in pkg.sphattn_gated_ffn_bwd(X, Wg, Wu, torch.zeros_like(dH), "gelu"):
        assert (t == 0).all()
    dH[:, 3:] = 0
    _, dWg, dWu = pkg.sphattn_gated_ffn_bwd(X, Wg, Wu, dH, "silu", want_dX=False)
    assert (dWg[3:] == 0).all() and (dWu[3:] == 0).all()
    for got, (want, tol) in zip((dWg, dWu), _units(X, Wg, Wu, dH, "silu")):
        _near(got, want, tol, "units")

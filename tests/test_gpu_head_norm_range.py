"""Norms of heads whose squares fp32 does not hold: a row times a power of two has, without eps or with one times its square, the same norm bit by bit."""
import pytest
import torch

from test_gpu_head_norm_rotary import _angle, _case, _exact

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.fixture(scope="module")
def pkg():
    import paper_2505_09326_amd as p
    p.load_library()
    return p


def _two_to(powers):
    """Exactly (the device's power function is not)."""
    return torch.tensor([2.0 ** p for p in powers.flatten().tolist()], dtype=torch.float32).view(powers.shape).to(DEV)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("B,N,H", [(1, 1, 16), (2, 333, 5), (1, 3000, 2)])
def test_powers_of_two(pkg, B, N, H, d, dtype):
    Xq, Xk, wq, wk, dQ, dK, positions, inv_freq, _ = _case(B, N, H, H, d, dtype, 1, torch.int64, d + N)
    g = torch.Generator(device=DEV).manual_seed(N)
    kw = dict(positions=positions, inv_freq=inv_freq, eps=0.0)
    want = *pkg.sphattn_head_norm_rotary_fwd(Xq, Xk, wq, wk, **kw), *pkg.sphattn_head_norm_rotary_bwd(Xq, Xk, wq, wk, dQ, dK, **kw)
    powers = [torch.tensor([0, 40, 50, 63, 64, 65, 80, 100, -40, -47, -48, -49, -60, -80, -100], device=DEV)[torch.randint(15, (B, N, H, 1), generator=g, device=DEV)] for _ in range(2)]
    times = lambda x, p: (x.float() * _two_to(p)).to(x.dtype)
    far = [times(x, p) for x, p in zip((Xq, Xk), powers)]
    got = *pkg.sphattn_head_norm_rotary_fwd(*far, wq, wk, **kw), *pkg.sphattn_head_norm_rotary_bwd(*far, wq, wk, dQ, dK, **kw)
    for i in (0, 1, 4, 5):                                     # Q, K, dwq, dwk
        assert torch.equal(got[i], want[i]), i
    for i, p in zip((2, 3), powers):                           # the rows' gradients have the other power (those that fp32 has as normal numbers)
        there = want[i].double() * _two_to(-p).double()
        kept = (there.abs() > 2.0 ** -120) & (there.abs() < 2.0 ** 127)
        assert kept.float().mean() > 0.9 and torch.equal(got[i].double()[kept], there[kept]), i


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_a_small_eps_counts(pkg, dtype):
    Xq, _, wq, *_ = _case(2, 50, 3, 0, 64, dtype, 0, torch.int64, 2)
    want = pkg.sphattn_head_norm_rotary_fwd(Xq, None, wq, eps=1.0)[0]
    for power in (-45, -55, -70):
        assert torch.equal(pkg.sphattn_head_norm_rotary_fwd((Xq.float() * 2.0 ** power).to(Xq.dtype), None, wq, eps=2.0 ** (2 * power))[0], want)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_elements_of_very_different_size(pkg, dtype):
    """One element of 1e30 among others of 1 and of 1e25: the formula in 64 bits to (64 / 2 + 10) 2^-24, as for every row, and the rounding."""
    g = torch.Generator(device=DEV).manual_seed(3)
    t = torch.float32 if dtype == "f32" else torch.bfloat16
    x = torch.randn(1, 9, 2, 64, generator=g, device=DEV)
    x[..., 3], x[..., 40:50] = 1e30, x[..., 40:50] * 1e25
    x[0, 4] = torch.randn(2, 64, generator=g, device=DEV) * 1e-30
    x[0, 5] = 0
    x = x.to(t)
    got = pkg.sphattn_head_norm_rotary_fwd(x, eps=1e-30)[0].double()
    v = x.double()
    want = (v / (v.square().mean(-1, keepdim=True) + float(torch.tensor(1e-30).float())).sqrt()).transpose(1, 2)
    assert ((got - want).abs() <= (42 * 2.0 ** -24 + torch.finfo(t).eps / 2 * (1 + 2.0 ** -7)) * want.abs() + 2.0 ** -126).all()
    assert (got[0, :, 5] == 0).all()
    # zeros without eps and rows that are not finite are what the formula makes of them
    x[0, 6, 0, 7], x[0, 7, 1, 9] = float("inf"), float("nan")
    got = pkg.sphattn_head_norm_rotary_fwd(x, eps=0.0)[0]
    assert got[0, :, 5].isnan().all() and got[0, 0, 6, 7].isnan() and (got[0, 0, 6, :7] == 0).all() and got[0, 1, 7].isnan().all() and got[0, 1, 6].isfinite().all()


@pytest.mark.parametrize("seed", [1, 2, 3])
def test_weights_gradients_over_many_rows(pkg, seed):
    """Sums over 54081 and 18027 rows in fp32.  Of each sum's norm: its terms' roundings, six of 0.29 2^-24 each in the mean (x r, the product with dy and dy's rotation), 0.7 2^-24; adding them, a
    chain of nine heads and five levels of lanes and waves, 0.29 2^-24 of what is there at each, sqrt(14) of them, 1.1; the angles' 2^-26 of a turn, 0.5; in fp64 behind that and the
    result's rounding, 0.3.  Together 1.5 2^-24 in the mean, and this asks for 2.7."""
    B, N, Hq, Hk, d = 3, 2003, 9, 3, 64
    Xq, Xk, wq, wk, dQ, dK, positions, inv_freq, sections = _case(B, N, Hq, Hk, d, "f32", 3, torch.int64, seed)
    grads = pkg.sphattn_head_norm_rotary_bwd(Xq, Xk, wq, wk, dQ, dK, positions, inv_freq, sections, True)
    angle = _angle(positions, inv_freq, sections, B, N)
    for got, x, w, g in ((grads[2], Xq, wq, dQ), (grads[3], Xk, wk, dK)):
        want = _exact(x, w, angle, True, True, float(torch.tensor(1e-6).float()), g)[2]
        assert float((got.double() - want).norm() / want.norm()) < 2.7 * 2.0 ** -24

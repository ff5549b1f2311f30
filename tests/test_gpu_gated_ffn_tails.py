"""The tail of gelu in 16 bits against the formula in 64 bits, each value to its own size: brought up by U it is what H and the gradients consist of.

A and U are one exact product each.  Tolerances (e = eps / 2 of the storage type): the share below A is off by 1.5e-5 of itself, its exponential's argument A^2 / 2 is rounded twice in
base 2, 2 u A^2 / 2 of it with u = 2^-24 and A = 13 at most, 1e-5: f = 3e-5 of the share and of A times the density, and the rounding e of H, of dA or dB and of the sum; fp16: half
a step below its normal numbers, 2^-25, of dA and dB as they are scaled, to 2^13 .. 2^14 of what the norms allow: 2^-24 here."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.fixture(scope="module")
def pkg():
    import paper_2505_09326_amd as p
    p.load_library()
    return p


@pytest.mark.parametrize("dtype,least", [(torch.bfloat16, -12.9), (torch.float16, -9.0)])
@pytest.mark.parametrize("T", [1, 20, 100, 700])
def test_gelu_tail(pkg, T, dtype, least):
    e, f, big = torch.finfo(dtype).eps / 2, 3e-5, 16384.0
    A = torch.linspace(least, 0.0, 500, device=DEV).to(dtype)
    X, Wg, Wu = torch.zeros(T, 8, device=DEV, dtype=dtype), torch.zeros(500, 8, device=DEV, dtype=dtype), torch.zeros(500, 8, device=DEV, dtype=dtype)
    X[:, 0], Wg[:, 0], Wu[:, 0] = 1, A, big
    a = A.double()
    below, density = 0.5 * torch.special.erfc(-a * math.sqrt(0.5)), torch.exp(-0.5 * a * a) / math.sqrt(2 * math.pi)
    step = 2.0 ** -25 if dtype == torch.float16 else 0.0
    H = pkg.sphattn_gated_ffn_fwd(X, Wg, Wu, "gelu").double()
    want = a * below * big
    assert ((H - want).abs() <= (e * (1 + 2.0 ** -10) + f) * want.abs() + step).all(), ((H / want - 1).abs().max(), A[((H / want - 1).abs()).nan_to_num().amax(0).argmax()])
    dH = torch.zeros(T, 500, device=DEV, dtype=dtype)
    dH[T // 2] = 1
    _, dWg, dWu = pkg.sphattn_gated_ffn_bwd(X, Wg, Wu, dH, "gelu", want_dX=False)
    slope = below + a * density
    for got, want, size in ((dWg[:, 0], big * slope, big * (below + a.abs() * density)), (dWu[:, 0], a * below, a.abs() * below)):
        assert ((got.double() - want).abs() <= 2 * e * (1 + 2.0 ** -7) * want.abs() + f * size + 2 * step + (2.0 ** -24 if step else 0.0)).all(), (got, want)

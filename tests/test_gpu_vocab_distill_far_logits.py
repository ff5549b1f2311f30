"""A teacher's logits far from 0 and far from each other, at small and large temperatures: what a row's logits have in common changes nothing, bit by bit, and what is far below the largest
has no part."""
import math

import pytest
import torch

from test_gpu_vocab_distill import _exact, _inputs, _near

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.fixture(scope="module")
def pkg():
    import paper_2505_09326_amd as p
    p.load_library()
    return p


def _all(pkg, X, W, ids, teacher, tau):
    losses, lse, kept = pkg.sphattn_vocab_distill_fwd(X, W, ids, teacher, 1.0, tau, keep=True)
    return losses, lse, kept, *pkg.sphattn_vocab_distill_bwd(X, W, ids, teacher, lse, kept, torch.ones_like(losses), 1.0, tau)


@pytest.mark.parametrize("tau", [1.0, 0.3, 0.01, 7.0])
@pytest.mark.parametrize("K", [3, 64, 200])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_common_offset_changes_nothing(pkg, K, tau, dtype):
    """The logits are multiples of 2^-8, so that each has its offset added without rounding."""
    X, W, ids, teacher, g = _inputs(90, 700, 64, K, dtype, K, 0.9)
    teacher = (teacher * 16 * tau).round() / 256
    offset = torch.randint(-16000, 16000, (90, 1), generator=g, device=DEV).float()
    shifted = teacher + offset
    assert torch.equal(torch.where(shifted.isfinite(), shifted - offset, teacher).nan_to_num(), teacher.nan_to_num())
    for a, b in zip(_all(pkg, X, W, ids, teacher, tau), _all(pkg, X, W, ids, shifted, tau)):
        assert torch.equal(a, b)


@pytest.mark.parametrize("tau,size", [(2.0 ** -20, 1.0), (2.0 ** -20, 1e33), (1.0, 1e38), (0.25, 3e38), (2.0 ** 20, 1e5), (2.0 ** 20, 1e12)])
@pytest.mark.parametrize("K", [5, 130])
def test_logits_of_any_size(pkg, tau, size, K):
    """Tolerances are those of the formulas with the largest logit's own distance to the others in the place of their size: in p what is further below it than 104 is 0."""
    X, W, ids, _, g = _inputs(40, 300, 48, K, "f32", 11 + K, 1.0)
    scale = min(1.0, tau)                                      # (so that the student's logits stay numbers)
    teacher = (torch.rand(40, K, generator=g, device=DEV) * 2 - 1) * size
    teacher[:, 1] = teacher[:, 0]                              # (two alike: where they are the largest each has half)
    ids[:, :2] = torch.tensor([7, 123], device=DEV)
    ids[5] = -1
    ids[5, 2] = 33                                             # one entry, far below 0
    teacher[5, 2] = -size
    best = torch.where(ids >= 0, teacher, -math.inf).amax(1, keepdim=True)
    near = torch.where(ids >= 0, teacher.double() - best.double(), 0.0)
    near = torch.where(near > -110.0 * tau, near, -math.inf).float()
    losses, lse, kept = pkg.sphattn_vocab_distill_fwd(X, W, ids, teacher, scale, tau, keep=True)
    (want, tol), (want_lse, tol_lse) = _exact(X, W, ids, near, scale, tau)
    _near(losses, want, tol, "losses")
    _near(lse, want_lse, tol_lse, "lse")
    g = torch.ones_like(losses)
    got = pkg.sphattn_vocab_distill_bwd(X, W, ids, teacher, lse, kept, g, scale, tau)
    for name, a, (w, t) in zip(("dX", "dW"), got, _exact(X, W, ids, near, scale, tau, g)):
        _near(a, w, t, name)

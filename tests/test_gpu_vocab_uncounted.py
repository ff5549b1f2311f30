"""Rows that do not count have no gradient, whatever comes back to the loss: an overflowed loss scale, or a NaN from further up."""
import pytest
import torch

from test_gpu_vocab_loss import DEV, _inputs

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def pkg():
    import paper_2505_09326_amd as p
    p.load_library()
    return p


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("T", [40, 200, 1500])
@pytest.mark.parametrize("dloss", [float("inf"), float("-inf"), float("nan")])
def test_rows_that_do_not_count_have_no_gradient(pkg, T, dtype, dloss):
    X, W, targets = _inputs(T, 500, 48, dtype, 1, 0.5)
    lse = pkg.sphattn_vocab_loss_fwd(X, W, targets)[1]
    for reduction in ("none", "sum", "mean"):
        back = torch.full((T,) if reduction == "none" else (), dloss, device=DEV)
        dX, dW = pkg.sphattn_vocab_loss_bwd(X, W, targets, lse, back, reduction=reduction)
        assert bool((dX[targets < 0] == 0).all()), reduction
        assert not bool(dX[targets >= 0].isfinite().any()) and not bool(dW.isfinite().any()), reduction

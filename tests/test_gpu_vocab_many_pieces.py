"""Gradients that are formed in two to five pieces of the vocabulary: sums of dX that go on from piece to piece, ids behind a piece's border.  How many pieces
a case has follows from the limits that stand in the source, so that a case which another limit makes one piece of fails here."""
import os
import re

import pytest
import torch

from paper_2505_09326_amd._build import CSRC
from test_gpu_vocab_f32 import _check, _inputs as f32_inputs
from test_gpu_vocab_loss import DEV, Exact, _inputs, _near

SOURCE = open(os.path.join(CSRC, "sphattn_train.hip")).read()


def pieces(T, V, D, dtype):
    """As vocab_bwd_plan cuts: whole pieces of 256 ids, G at most kOnePieceBytes in one or kPieceBytes (or X's size) in each of several, 2^18 ids at most."""
    limits = re.search(r"kPieceBytes = (\d+)u << 20, kOnePieceBytes = (\d+)u << 20;", SOURCE)
    several, one = (int(x) << 20 for x in limits.groups())
    parts = 1 if dtype != "f32" else 2 if T <= 64 else 3
    row_bytes = 2 * parts * T
    limit = max(one if row_bytes * V <= one else several, row_bytes * -(-D // 8) * 8)
    most = min(max(limit // row_bytes // 256 * 256, 256), 1 << 18)
    n = -(-V // most)
    piece = -(-(-(-V // n)) // 256) * 256
    return -(-V // piece)


CASES = [  # T, V, D, dtype, share of rows that count, pieces
    (6000, 18100, 24, "bf16", 1.0, 1), (8192, 27001, 24, "bf16", 0.7, 2), (8192, 52003, 40, "f16", 0.1, 4), (7000, 31007, 72, "f16", 1.0, 2),
    (40, 300_001, 16, "bf16", 1.0, 2), (8000, 60001, 16, "bf16", 0.3, 4),
]
F32_CASES = [(1500, 30000, 40, 1), (6000, 18100, 36, 3), (4000, 21003, 20, 2), (1200, 200_003, 8, 6), (64, 270_000, 12, 2)]


def test_the_cases_have_the_pieces_that_they_are_here_for():
    for T, V, D, dtype, _, n in CASES:
        assert pieces(T, V, D, dtype) == n, (T, V, D, dtype)
    for T, V, D, n in F32_CASES:
        assert pieces(T, V, D, "f32") == n, (T, V, D)


@pytest.fixture(scope="module")
def pkg():
    import paper_2505_09326_amd as p
    p.load_library()
    yield p
    # what the 64-bit products left in the allocator is no memory of later tests
    torch._C._cuda_clearCublasWorkspaces()
    torch.cuda.empty_cache()


@pytest.mark.gpu
@pytest.mark.parametrize("T,V,D,dtype,share,n", CASES)
def test_pieces(pkg, T, V, D, dtype, share, n):
    X, W, targets = _inputs(T, V, D, dtype, 43, share)
    targets[0] = V - 1
    dloss = torch.tensor(2.0 if dtype != "f16" else 256.0, device=DEV)
    want = Exact(X, W, targets, 1.0, dloss, "mean")
    lse = pkg.sphattn_vocab_loss_fwd(X, W, targets, reduction="mean", all_rows=False)[1]
    dX, dW = pkg.sphattn_vocab_loss_bwd(X, W, targets, lse, dloss, reduction="mean")
    _near(dX, want.dX, want.dX_tol, "dX")
    _near(dW, want.dW, want.dW_tol, "dW")
    assert bool((dX[targets < 0] == 0).all())
    again = pkg.sphattn_vocab_loss_bwd(X, W, targets, lse, dloss, reduction="mean")
    assert torch.equal(dX, again[0]) and torch.equal(dW, again[1])


@pytest.mark.gpu
@pytest.mark.parametrize("T,V,D,n", F32_CASES)
def test_pieces_of_fp32(pkg, T, V, D, n):
    X, W, targets, _ = f32_inputs(T, V, D, 44)
    _check(pkg, X, W, targets, 1.0)

"""Clipping by the common norm against 64 bits.  The norm is summed in fp64 and rounded once to fp32 (2^-24, and some 2^-50 of the sum); the
factor is rounded to fp32 (2^-24) and the product to the storage type."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U32 = 2.0 ** -24


@pytest.fixture(scope="module")
def pkg():
    import paper_2505_09326_amd as p
    p.load_library()
    return p


def _tensors(sizes, dtypes, seed, spread=3, offset=0):
    g = torch.Generator().manual_seed(seed)
    out = []
    for i, n in enumerate(sizes):
        x = torch.randn(n, generator=g) * 10.0 ** (i % spread - 1)
        t = dtypes[i % len(dtypes)]
        out.append(torch.empty(n + offset, dtype=t, device=DEV)[offset:].copy_(x.to(t)))
    return out


def _check(grads, outs, norm, limit):
    want = math.sqrt(math.fsum(float((x.double() ** 2).sum()) for x in grads))
    assert float(norm) == pytest.approx(want, rel=2 * U32)
    f = min(1.0, limit / (want + 1e-6))
    for x, y in zip(grads, outs):
        ref = x.double() * f
        tol = (torch.finfo(x.dtype).eps / 2 + 3 * U32) * ref.abs() + torch.finfo(x.dtype).tiny * torch.finfo(x.dtype).eps
        assert bool(((y.double() - ref).abs() <= tol).all())


F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
CASES = [  # sizes, types, offset in elements
    ([1], [F32], 0), ([5], [BF16], 0), ([8192], [F16], 0), ([8193, 1, 8191], [F32], 0), ([1000] * 7, [F32, BF16, F16], 0),
    ([0, 17, 0, 0, 300, 0], [BF16], 0), ([12345, 777, 64], [F16, F32], 1), ([100_003, 3], [BF16], 3),
    (list(range(1, 260)), [F32, BF16], 0),         # three launches' worth of tensors
    ([9_000_001, 50], [BF16], 0),                  # more pieces than workgroups
]


@pytest.mark.parametrize("sizes,types,offset", CASES)
@pytest.mark.parametrize("limit", [0.5, 1e9])
def test_norm_and_scaling(pkg, sizes, types, offset, limit):
    grads = _tensors(sizes, types, len(sizes) + sizes[0], offset=offset)
    before = [x.clone() for x in grads]
    outs = [torch.full_like(x, 3.0) for x in grads]
    norm = pkg.sphattn_clip_grads(grads, limit, out=outs)
    _check(before, outs, norm, limit)
    assert all(torch.equal(x, y) for x, y in zip(grads, before))
    again = pkg.sphattn_clip_grads(grads, limit)   # in place
    assert float(again) == float(norm)
    assert all(torch.equal(x, y) for x, y in zip(grads, outs))


def test_values_at_the_ends_of_the_range(pkg):
    big, small = torch.full((3000,), 2e38, device=DEV), torch.full((5000,), 1e-38, device=DEV)
    assert float(pkg.sphattn_clip_grads([small], 1.0)) == pytest.approx(1e-38 * math.sqrt(5000), rel=1e-5)
    out = [torch.empty_like(big)]
    norm = pkg.sphattn_clip_grads([big], 1.0, out=out)
    assert float(norm) == float("inf")             # the norm is past fp32; the gradients are scaled by it all the same
    assert bool(((out[0] - 1 / math.sqrt(3000)).abs() <= 1e-6).all())


def test_what_is_not_finite(pkg):
    x = [torch.ones(100, device=DEV), torch.tensor([float("inf"), 1.0], device=DEV)]
    out = [torch.empty_like(t) for t in x]
    assert float(pkg.sphattn_clip_grads(x, 1.0, out=out)) == float("inf")
    assert bool((out[0] == 0).all()) and bool(out[1][0].isnan()) and float(out[1][1]) == 0
    x[1][0] = float("nan")
    assert math.isnan(float(pkg.sphattn_clip_grads(x, 1.0, out=out)))
    assert all(bool(t.isnan().all()) for t in out)


def test_zero_limit_zero_gradients_and_none(pkg):
    x = [torch.ones(9, device=DEV)]
    assert float(pkg.sphattn_clip_grads(x, 0.0)) == 3.0 and bool((x[0] == 0).all())
    assert float(pkg.sphattn_clip_grads(x, 1.0)) == 0.0 and bool((x[0] == 0).all())
    assert float(pkg.sphattn_clip_grads([], 1.0, norm=torch.full((), 5.0, device=DEV))) == 0.0


def test_dense_tensors_of_any_order(pkg):
    x = torch.randn(30, 50, device=DEV).t()
    y = torch.randn(4, 6, 5, 3, device=DEV).to(memory_format=torch.channels_last)
    before = [x.clone(), y.clone()]
    norm = pkg.sphattn_clip_grads([x, y], 1.0)
    _check([t.contiguous() for t in before], [x.contiguous(), y.contiguous()], norm, 1.0)
    with pytest.raises(ValueError):
        pkg.sphattn_clip_grads([torch.randn(10, 10, device=DEV)[:, :5]], 1.0)
    with pytest.raises(ValueError):
        pkg.sphattn_clip_grads([torch.randn(1, 10, device=DEV).expand(5, 10)], 1.0)


def test_graph(pkg):
    grads = _tensors([5000, 33], [F32, BF16], 3)
    outs = [torch.empty_like(t) for t in grads]
    pkg.sphattn_clip_grads(grads, 1.0, out=outs)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        norm = pkg.sphattn_clip_grads(grads, 1.0, out=outs)
    for turn in range(3):
        for t in grads:
            t.mul_(1.0 + turn)
        for t in outs:
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        _check(grads, outs, norm, 1.0)

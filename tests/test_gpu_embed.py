"""Embedding lookup with scaling and the gradient of its table against the formulas in 64 bits.

Tolerances, from the roundings: the factor scale * mult and its product with an element are rounded to fp32 (2^-24 each), the result
once to the storage type (eps / 2).  The gradient adds n products in fp32: at most (n + 2) 2^-24 of the sum of their
magnitudes, and eps / 2 of the result."""
import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U32 = 2.0 ** -24
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


@pytest.fixture(scope="module")
def pkg():
    import paper_2505_09326_amd as p
    p.load_library()
    return p


def _half_step(t):
    return torch.finfo(t).eps / 2


def _tiny(t):
    return torch.finfo(t).tiny * torch.finfo(t).eps      # the smallest subnormal


def _tokens(T, V, kind, g):
    if kind == "one":
        return torch.full((T,), V - 1, dtype=torch.int64)
    x = torch.randint(V, (T,), generator=g)
    if kind == "heavy":
        x[torch.rand(T, generator=g) < 0.6] = V // 2
    if kind == "gaps":                             # negative: no token
        x[torch.rand(T, generator=g) < 0.3] = -1
    if kind == "none":
        x[:] = -7
    return x


def _case(T, V, D, dtype, kind, mult, seed, ids=torch.int64, offset=0):
    g = torch.Generator().manual_seed(seed)
    t = TYPES[dtype]

    def make(rows):
        flat = torch.empty(rows * D + offset, dtype=t, device=DEV)[offset:]      # offset: rows that begin between 16-byte borders
        return flat.copy_(torch.randn(rows * D, generator=g).to(t)).view(rows, D)
    tokens = _tokens(T, V, kind, g).to(ids).to(DEV)
    m = torch.poisson(torch.full((T,), 1.5), generator=g).to(DEV) if mult else None
    return tokens, make(V), make(T), m


def _reference(tokens, table, dO, mult, scale):
    V = table.shape[0]
    live = (tokens >= 0) & (tokens < V)
    f = torch.full((tokens.numel(),), scale, dtype=torch.float64, device=DEV)
    if mult is not None:
        f = f * mult.double()
    at = tokens.long().clamp(0, V - 1)
    out = table.double()[at] * f[:, None] * live[:, None]
    terms = dO.double() * (f * live)[:, None]
    grad, size = (torch.zeros(table.shape, dtype=torch.float64, device=DEV) for _ in range(2))
    grad.index_add_(0, at, terms)
    size.index_add_(0, at, terms.abs())
    n = torch.zeros(V, dtype=torch.float64, device=DEV).index_add_(0, at, live.double())
    return out, grad, size, n


SHAPES = [  # T, V, D, dtype, tokens, mult, id type, offset
    (1, 1, 1, "f32", "one", False, torch.int64, 0),
    (1, 300, 64, "bf16", "even", True, torch.int32, 0),
    (7, 3, 5, "f16", "even", True, torch.int64, 0),
    (65, 40, 129, "bf16", "gaps", True, torch.int64, 0),
    (200, 513, 264, "f32", "even", False, torch.int32, 0),
    (1000, 77, 96, "bf16", "heavy", True, torch.int64, 0),
    (1000, 77, 96, "bf16", "heavy", True, torch.int64, 3),
    (3001, 2000, 515, "f16", "heavy", False, torch.int64, 0),
    (4096, 5003, 512, "f32", "one", True, torch.int64, 0),
    (5000, 200000, 24, "bf16", "even", False, torch.int64, 0),       # more ids than 256 workgroups of 512
    (40000, 900, 72, "bf16", "heavy", True, torch.int32, 0),         # pieces of 32 positions
    (40000, 900, 40, "f32", "one", False, torch.int64, 0),           # one run over all of them
    (333, 50, 16, "f16", "none", False, torch.int64, 0),
]


@pytest.mark.parametrize("T,V,D,dtype,kind,mult,ids,offset", SHAPES)
def test_rows_and_gradient(pkg, T, V, D, dtype, kind, mult, ids, offset):
    tokens, table, dO, m = _case(T, V, D, dtype, kind, mult, 3 + T + V, ids, offset)
    t, scale = TYPES[dtype], 1.0 / 3.0
    want, grad, size, n = _reference(tokens, table, dO, m, scale)
    O = pkg.sphattn_embed_fwd(tokens, table, m, scale)
    err = (O.double() - want).abs()
    assert bool((err <= (_half_step(t) + 3 * U32) * want.abs() + _tiny(t)).all())
    G = pkg.sphattn_embed_bwd(tokens, dO, V, m, scale)
    err = (G.double() - grad).abs()
    assert bool((err <= _half_step(t) * grad.abs() + (n[:, None] + 3) * U32 * size + _tiny(t)).all())
    assert bool((G[n == 0] == 0).all())
    again = pkg.sphattn_embed_bwd(tokens, dO, V, m, scale)
    assert torch.equal(G.view(torch.uint8), again.view(torch.uint8))   # (bits)


def test_tokens_that_are_none_or_too_large(pkg):
    table = torch.randn(9, 40, device=DEV).bfloat16()
    for ids in (torch.int32, torch.int64):
        tokens = torch.tensor([3, -1, 9, 8, 2 ** 31 - 1, -2 ** 31], device=DEV).to(ids)
        O = pkg.sphattn_embed_fwd(tokens, table).float()
        assert torch.equal(O[[0, 3]], table[[3, 8]].float())
        assert bool((O[[1, 5]] == 0).all()) and bool(O[[2, 4]].isnan().all())
        G = pkg.sphattn_embed_bwd(tokens, torch.ones(6, 40, device=DEV, dtype=torch.bfloat16), 9)
        assert bool((G[[3, 8]] == 1).all()) and int((G != 0).sum()) == 80
    tokens = torch.tensor([2 ** 32 + 3, -2 ** 40, 2 ** 62], device=DEV)   # not to be taken for their lower halves
    O = pkg.sphattn_embed_fwd(tokens, table).float()
    assert bool(O[[0, 2]].isnan().all()) and bool((O[1] == 0).all())


def test_nan_and_inf_stay_in_their_rows(pkg):
    g = torch.Generator().manual_seed(5)
    dO = torch.randn(300, 72, generator=g).to(DEV)
    tokens = torch.randint(20, (300,), generator=g).to(DEV)
    dO[tokens == 4] = float("nan")
    dO[(tokens == 5).nonzero()[0], 7] = float("inf")
    G = pkg.sphattn_embed_bwd(tokens, dO, 20)
    bad = ~G.isfinite()
    assert bool(bad[4].all()) and bool(bad[5, 7]) and int(bad.sum()) == 73


def test_no_tokens(pkg):
    empty = torch.empty(0, dtype=torch.int64, device=DEV)
    assert pkg.sphattn_embed_fwd(empty, torch.ones(4, 8, device=DEV)).shape == (0, 8)
    G = pkg.sphattn_embed_bwd(empty, torch.empty(0, 8, device=DEV), 4, dtable=torch.full((4, 8), 3.0, device=DEV))
    assert bool((G == 0).all())


def test_autograd(pkg):
    from paper_2505_09326_amd.autograd import token_embedding
    tokens, table, dO, m = _case(60, 31, 48, "f32", "gaps", True, 11)
    table.requires_grad_(True)
    shaped, weights = tokens.view(3, 20), m.view(3, 20)
    out = token_embedding(shaped, table, weights, 2.0)
    assert out.shape == (3, 20, 48)
    grad, = torch.autograd.grad(out, table, dO.view(3, 20, 48))
    # against differences: the map is linear in the table
    g = torch.Generator().manual_seed(1)
    step = torch.randn(31, 48, generator=g).to(DEV)
    with torch.no_grad():
        change = (token_embedding(shaped, step, weights, 2.0).double() * dO.view(3, 20, 48).double()).sum()
    assert float((grad.double() * step.double()).sum() - change) == pytest.approx(0, abs=60 * 48 * 4 * U32 * float((grad.abs() * step.abs()).sum()))


def test_other_stream_and_graph(pkg):
    tokens, table, dO, m = _case(500, 90, 80, "bf16", "heavy", True, 21)
    want_O, want_G = pkg.sphattn_embed_fwd(tokens, table, m), pkg.sphattn_embed_bwd(tokens, dO, 90, m)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        G = pkg.sphattn_embed_bwd(tokens, dO, 90, m)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(G, want_G)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        O, G = pkg.sphattn_embed_fwd(tokens, table, m), pkg.sphattn_embed_bwd(tokens, dO, 90, m)
    for turn in range(3):
        O.fill_(7.0)
        G.fill_(7.0)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(O, want_O) and torch.equal(G, want_G), turn
        tokens.copy_(tokens.roll(turn + 1))        # the next replay reads other tokens
        want_O, want_G = pkg.sphattn_embed_fwd(tokens, table, m), pkg.sphattn_embed_bwd(tokens, dO, 90, m)

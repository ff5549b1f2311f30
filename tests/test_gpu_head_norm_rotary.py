"""Norms of heads with the rotation by positions, forward and backward, against the formulas in 64 bits.

Tolerances (u = 2^-24, e = eps / 2 of the storage type):
  y        x r w: r's sum of d squares and its root (d / 2 + 8) u, two products 2 u
  angle    its fraction of a turn in fp32 and the function's own error 8 u, position times frequency in fp64 (here and there) 2^-50 of the angle
  o        (|y_a| + |y_b|) (y's + the angle's + 3 u) and the rounding, e |o|
  dy       the angle's + 3 u of the two gradients' sizes
  dw       dy's and x r's per term, and (heads + tokens of a lane + 120) u of the terms' sizes for adding them, e |dw|
  dx       r times (dy's |w| + (d + 24) u of |dn| and of |x r| mean |dn x r|), e |dx|
and half a step of the type's smallest number, 2^-149 in fp32, 2^-25 in fp16."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U = 2.0 ** -24
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
TINY = {"f32": 2.0 ** -149, "bf16": 2.0 ** -133, "f16": 2.0 ** -25}


@pytest.fixture(scope="module")
def pkg():
    import paper_2505_09326_amd as p
    p.load_library()
    return p


def _pairs(x, interleaved):
    return (x[..., 0::2], x[..., 1::2]) if interleaved else x.chunk(2, -1)


def _join(a, b, interleaved):
    return torch.stack((a, b), -1).flatten(-2) if interleaved else torch.cat((a, b), -1)


def _angle(positions, inv_freq, sections, B, N):
    """[B,N,1,d/2]; None without positions."""
    if positions is None:
        return None
    at = positions.double()
    at = at.expand(B, N)[None] if at.dim() < 3 else at.expand(at.shape[0], B, N)
    sections = sections or [inv_freq.numel()]
    axis = torch.repeat_interleave(torch.arange(len(sections), device=DEV), torch.tensor(sections, device=DEV))
    return (at[axis].permute(1, 2, 0) * inv_freq.double())[:, :, None]


def _exact(x, w, angle, interleaved, norm, eps, dO=None):
    """o [B,H,N,d] and its tolerance without the rounding, and with dO (dx, tolerance, dw, tolerance per term)."""
    x, d = x.double(), x.shape[-1]
    w = torch.ones(d, dtype=torch.float64, device=DEV) if w is None else w.double()
    r = (x.square().mean(-1, keepdim=True) + eps).rsqrt() if norm else torch.ones_like(x[..., :1])
    n, ty = x * r, (d / 2 + 10) * U
    cos, sin, ta = (1.0, 0.0, 0.0) if angle is None else (angle.cos(), angle.sin(), 11 * U + 2.0 ** -50 * angle.abs())
    a, b = _pairs(n * w, interleaved)
    o = _join(a * cos - b * sin, b * cos + a * sin, interleaved)
    size = a.abs() + b.abs()
    tol = _join(size * (ty + ta), size * (ty + ta), interleaved)
    if dO is None:
        return o.transpose(1, 2), tol.transpose(1, 2)
    a, b = _pairs(dO.double().transpose(1, 2), interleaved)
    dy = _join(a * cos + b * sin, b * cos - a * sin, interleaved)
    tdy = _join((a.abs() + b.abs()) * ta, (a.abs() + b.abs()) * ta, interleaved)
    dn = dy * w
    m, mm = (dn * n).mean(-1, keepdim=True), (dn * n).abs().mean(-1, keepdim=True) + (tdy * w.abs() * n.abs()).mean(-1, keepdim=True) / U
    dx = r * (dn - n * m) if norm else dn
    tdx = r * (tdy * w.abs() + (d + 24) * U * dn.abs() + (n.abs() * (d + 24) * U * mm if norm else 0.0))
    return dx, tdx, (dy * n).sum((0, 1, 2)), ((tdy + dy.abs() * (d / 2 + 10) * U) * n.abs()).sum((0, 1, 2)), (dy * n).abs().sum((0, 1, 2))


def _near(got, want, tol, dtype, what):
    off = (got.double() - want).abs()
    allowed = tol + torch.finfo(TYPES[dtype]).eps / 2 * want.abs() * (1 + 2.0 ** -10) + TINY[dtype] + tol * torch.finfo(TYPES[dtype]).eps
    bad = off > allowed
    assert not bad.any(), f"{what}: {int(bad.sum())} of {bad.numel()}, worst {float((off / allowed.clamp_min(1e-300)).max()):.2f} of its tolerance"


def _freq(d, base=10000.0):
    return torch.pow(base, -torch.arange(0, d, 2, device=DEV, dtype=torch.float64) / d).float()


def _case(B, N, Hq, Hk, d, dtype, axes, ids, seed, far=0):
    g = torch.Generator(device=DEV).manual_seed(seed)
    r = lambda *s: torch.randn(s, generator=g, device=DEV)
    packed = (r(B, N, (Hq + 2 * max(Hk, 1)) * d) * (0.2 + torch.rand((B, N, 1), generator=g, device=DEV))).to(TYPES[dtype])
    Xq = packed[..., :Hq * d].view(B, N, Hq, d)
    Xk = packed[..., Hq * d:(Hq + Hk) * d].view(B, N, Hk, d) if Hk else None
    wq, wk = (1 + 0.3 * r(d)).to(TYPES[dtype]), (1 + 0.3 * r(d)).to(TYPES[dtype]) if Hk else None
    dQ, dK = r(B, Hq, N, d).to(TYPES[dtype]), r(B, Hk, N, d).to(TYPES[dtype]) if Hk else None
    if axes == 0:
        return Xq, Xk, wq, wk, dQ, dK, None, None, None
    positions = torch.randint(-5, 300, (axes, B, N), generator=g, device=DEV) + far
    sections = {1: [d // 2], 2: [d // 2 - 9, 9], 3: [16, 0, d // 2 - 16]}[axes]
    positions = (positions[0] if axes == 1 else positions).to(ids)
    return Xq, Xk, wq, wk, dQ, dK, positions, _freq(d), sections


CASES = [  # B, N, Hq, Hk, d, dtype, axes, ids, interleaved, norm, far
    (1, 1, 1, 0, 64, "f32", 1, torch.int64, False, True, 0),
    (1, 1, 16, 4, 128, "bf16", 1, torch.int64, False, True, 30000),
    (3, 1, 5, 5, 128, "f16", 1, torch.int32, True, True, 0),
    (2, 77, 7, 3, 64, "bf16", 3, torch.int64, True, True, 0),
    (2, 333, 4, 2, 128, "f32", 2, torch.int32, False, True, 0),
    (1, 1001, 3, 1, 64, "f16", 1, torch.int64, False, True, 1000000),
    (1, 130, 9, 3, 128, "f32", 1, torch.int64, True, True, 2 ** 31 + 12345),
    (5, 9, 33, 11, 64, "f32", 3, torch.int32, False, False, 0),
    (2, 50, 6, 6, 128, "bf16", 0, torch.int64, False, True, 0),
    (2, 50, 2, 1, 64, "f16", 0, torch.int64, False, False, 0),
    (2, 9001, 2, 1, 128, "bf16", 1, torch.int64, False, True, 0),
]


@pytest.mark.parametrize("B,N,Hq,Hk,d,dtype,axes,ids,interleaved,norm,far", CASES)
def test_forward_and_gradients(pkg, B, N, Hq, Hk, d, dtype, axes, ids, interleaved, norm, far):
    Xq, Xk, wq, wk, dQ, dK, positions, inv_freq, sections = _case(B, N, Hq, Hk, d, dtype, axes, ids, 7 * N + d + Hq, far)
    kw = dict(positions=positions, inv_freq=inv_freq, sections=sections, interleaved=interleaved, norm=norm, eps=1e-5)
    Q, K = pkg.sphattn_head_norm_rotary_fwd(Xq, Xk, wq, wk, **kw)
    grads = pkg.sphattn_head_norm_rotary_bwd(Xq, Xk, wq, wk, dQ, dK, **kw)
    assert (K is None) == (Hk == 0) and Q.is_contiguous() and Q.shape == (B, Hq, N, d)
    angle = _angle(positions, inv_freq, sections, B, N)
    lanes = B * N // (1024 * 16) + 1
    for i, (x, w, o, g, H) in enumerate(((Xq, wq, Q, dQ, Hq), (Xk, wk, K, dK, Hk))):
        if x is None:
            assert grads[i] is None and grads[2 + i] is None
            continue
        _near(o, *_exact(x, w, angle, interleaved, norm, 1e-5), dtype, f"o {i}")
        dx, tdx, dw, tdw, size = _exact(x, w, angle, interleaved, norm, 1e-5, g)
        _near(grads[i], dx, tdx, dtype, f"dx {i}")
        _near(grads[2 + i], dw, tdw + (H * lanes + lanes + 120) * U * size, dtype, f"dw {i}")
        assert grads[i].is_contiguous()
    again = (*pkg.sphattn_head_norm_rotary_fwd(Xq, Xk, wq, wk, **kw), *pkg.sphattn_head_norm_rotary_bwd(Xq, Xk, wq, wk, dQ, dK, **kw))
    for a, b in zip(again, (Q, K, *grads)):
        assert a is b is None or torch.equal(a, b)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
def test_places_in_a_cache_and_odd_strides(pkg, dtype):
    """Rows go where the strides say and nothing else is touched; rows that start anywhere; positions shared by the sequences."""
    B, N, H, d, cap = 3, 5, 4, 64, 23
    Xq, Xk, wq, wk, dQ, dK, positions, inv_freq, _ = _case(B, N, H, H, d, dtype, 1, torch.int64, 3)
    want = pkg.sphattn_head_norm_rotary_fwd(Xq, Xk, wq, wk, positions=positions[:1], inv_freq=inv_freq)
    cache = torch.full((B, H, cap, d), 7.0, device=DEV, dtype=TYPES[dtype])
    wide = torch.full((B, N, H, d + 3), 7.0, device=DEV, dtype=TYPES[dtype])          # rows of d + 3 elements, from the second on
    version = cache._version
    Q, K = pkg.sphattn_head_norm_rotary_fwd(Xq, Xk, wq, wk, positions=positions[0], inv_freq=inv_freq, Q=wide[..., 1:d + 1].transpose(1, 2), K=cache[:, :, 9:9 + N])
    assert cache._version > version
    assert torch.equal(K, want[1]) and torch.equal(cache[:, :, 9:9 + N], want[1]) and torch.equal(wide[..., 1:d + 1].transpose(1, 2), want[0])
    assert (cache[:, :, :9] == 7).all() and (cache[:, :, 9 + N:] == 7).all() and (wide[..., 0] == 7).all() and (wide[..., d + 1:] == 7).all()
    # inputs of odd strides, one row for every head and token, gradients into a packed buffer
    odd = torch.zeros((B, N, H, d + 3), device=DEV, dtype=TYPES[dtype])
    odd[..., 3:] = Xq
    assert torch.equal(pkg.sphattn_head_norm_rotary_fwd(odd[..., 3:], None, wq, positions=positions, inv_freq=inv_freq)[0],
                       pkg.sphattn_head_norm_rotary_fwd(Xq, None, wq, positions=positions, inv_freq=inv_freq)[0])
    one = Xq[:1, :1, :1].expand(B, N, H, d)
    assert torch.equal(pkg.sphattn_head_norm_rotary_fwd(one, None, wq, positions=positions, inv_freq=inv_freq)[0],
                       pkg.sphattn_head_norm_rotary_fwd(one.contiguous(), None, wq, positions=positions, inv_freq=inv_freq)[0])
    kw = dict(positions=positions, inv_freq=inv_freq)
    grads = pkg.sphattn_head_norm_rotary_bwd(Xq, Xk, wq, wk, dQ, dK, **kw)
    packed = torch.full((B, N, 3 * H * d), 7.0, device=DEV, dtype=TYPES[dtype])
    views = packed[..., :H * d].view(B, N, H, d), packed[..., H * d:2 * H * d].view(B, N, H, d)
    scattered = dQ.transpose(1, 2).contiguous().transpose(1, 2)
    got = pkg.sphattn_head_norm_rotary_bwd(Xq, Xk, wq, wk, scattered, dK, **kw, dXq=views[0], dXk=views[1])
    for a, b in zip(got, grads):
        assert torch.equal(a, b)
    assert (packed[..., 2 * H * d:] == 7).all()
    # one at a time
    only = pkg.sphattn_head_norm_rotary_bwd(Xq, Xk, wq, wk, dQ, dK, **kw, want_dX=(False, True), want_dw=(False, False))
    assert only[0] is only[2] is only[3] is None and torch.equal(only[1], grads[1])
    only = pkg.sphattn_head_norm_rotary_bwd(Xq, Xk, wq, wk, dQ, dK, **kw, want_dX=(False, False), want_dw=(True, False))
    assert only[0] is only[1] is only[3] is None and torch.equal(only[2], grads[2])


def test_rows_past_32_bits(pkg):
    """A cache in which a head's rows lie more than 2^31 elements behind the start."""
    B, N, H, d = 1, 2, 2, 128
    Xq, Xk, wq, wk, *_ = _case(B, N, H, H, d, "bf16", 0, torch.int64, 4)
    cap = (2 ** 31 + 2 ** 20) // d
    cache = torch.empty((B, H, cap, d), device=DEV, dtype=torch.bfloat16)
    _, want = pkg.sphattn_head_norm_rotary_fwd(Xq, Xk, wq, wk)
    pkg.sphattn_head_norm_rotary_fwd(Xq, Xk, wq, wk, K=cache[:, :, cap - 2:])
    assert torch.equal(cache[:, :, cap - 2:], want)
    again = pkg.sphattn_head_norm_rotary_fwd(cache[:, :, cap - 2:].transpose(1, 2), None, wk)[0]
    assert torch.equal(again, pkg.sphattn_head_norm_rotary_fwd(want.transpose(1, 2).contiguous(), None, wk)[0])


def test_empty_calls(pkg):
    for B, N in ((0, 5), (2, 0)):
        x, w = torch.zeros((B, N, 3, 64), device=DEV), torch.ones(64, device=DEV)
        Q, K = pkg.sphattn_head_norm_rotary_fwd(x, x, w, w, positions=torch.zeros((B, N), dtype=torch.int64, device=DEV), inv_freq=_freq(64))
        assert Q.shape == K.shape == (B, 3, N, 64)
        grads = pkg.sphattn_head_norm_rotary_bwd(x, x, w, w, Q, K)
        assert grads[0].shape == x.shape and (grads[2] == 0).all() and (grads[3] == 0).all()


def test_what_is_not_finite_stays_in_its_row(pkg):
    x, w = torch.randn(2, 6, 3, 128, device=DEV), torch.ones(128, device=DEV)
    clean = pkg.sphattn_head_norm_rotary_fwd(x, None, w, positions=torch.arange(6, device=DEV), inv_freq=_freq(128))[0]
    x[1, 2, 0, 5], x[0, 3, 1, 7] = float("nan"), float("inf")
    x[0, 0, 0] = 0                                             # a row of zeros has the norm sqrt(eps)
    got = pkg.sphattn_head_norm_rotary_fwd(x, None, w, positions=torch.arange(6, device=DEV), inv_freq=_freq(128))[0]
    hit = torch.zeros(2, 3, 6, dtype=torch.bool, device=DEV)
    hit[1, 0, 2] = hit[0, 1, 3] = hit[0, 0, 0] = True
    assert torch.equal(got[~hit], clean[~hit]) and got[1, 0, 2].isnan().all() and got[0, 1, 3].isnan().any() and (got[0, 0, 0] == 0).all()


def test_autograd_against_differences(pkg):
    """The gradients of a product with fixed directions, against central differences of the formula in 64 bits (step 2^-10: the third
    derivative's share is below 2^-16 of the largest gradient, and tests of the gradients themselves are tighter)."""
    from paper_2505_09326_amd import autograd
    B, N, Hq, Hk, d = 2, 5, 3, 1, 64
    Xq, Xk, wq, wk, dQ, dK, positions, inv_freq, sections = _case(B, N, Hq, Hk, d, "f32", 3, torch.int64, 11)
    leaves = [t.detach().clone().requires_grad_(True) for t in (Xq, Xk, wq, wk)]
    Q, K = autograd.head_norm_rotary(*leaves, positions, inv_freq, sections, True)
    ((Q * dQ).sum() + (K * dK).sum()).backward()
    angle = _angle(positions, inv_freq, sections, B, N)
    value = lambda xq, xk, a, b: float((_exact(xq, a, angle, True, True, 1e-6)[0] * dQ).sum() + (_exact(xk, b, angle, True, True, 1e-6)[0] * dK).sum())
    g = torch.Generator(device=DEV).manual_seed(5)
    at = [t.detach().double() for t in leaves]
    for i in range(4):
        step = torch.randn(at[i].shape, generator=g, device=DEV, dtype=torch.float64)
        step *= 2.0 ** -10 / step.norm()
        up, down = (value(*[t + s * step if j == i else t for j, t in enumerate(at)]) for s in (1, -1))
        slope = float((leaves[i].grad.double() * step).sum())
        assert abs((up - down) / 2 - slope) <= 2.0 ** -16 * float(leaves[i].grad.norm()) * float(step.norm()) + 1e-12, i
    with pytest.raises(RuntimeError):                          # no second derivative
        y = autograd.head_norm_rotary(*leaves)[0]
        first, = torch.autograd.grad(y.sum(), leaves[:1], create_graph=True)
        first.sum().backward()


def test_autograd_of_slices_of_a_projection(pkg):
    from paper_2505_09326_amd import autograd
    B, N, Hq, Hk, d = 2, 40, 4, 2, 64
    *_, dQ, dK, positions, inv_freq, sections = _case(B, N, Hq, Hk, d, "bf16", 1, torch.int32, 12)
    packed = torch.randn(B, N, (Hq + 2 * Hk) * d, device=DEV).bfloat16().requires_grad_(True)
    w = torch.randn(d, device=DEV).bfloat16().requires_grad_(True)
    split = lambda t: (t[..., :Hq * d].view(B, N, Hq, d), t[..., Hq * d:(Hq + Hk) * d].view(B, N, Hk, d))
    Q, K = autograd.head_norm_rotary(*split(packed), w, w, positions, inv_freq)        # one weight for both
    dp, dw = torch.autograd.grad((Q, K), (packed, w), (dQ, dK))
    want = pkg.sphattn_head_norm_rotary_bwd(*split(packed.detach()), w.detach(), w.detach(), dQ, dK, positions, inv_freq)
    assert torch.equal(split(dp)[0], want[0]) and torch.equal(split(dp)[1], want[1]) and (dp[..., (Hq + Hk) * d:] == 0).all()
    assert torch.equal(dw, want[2] + want[3])
    only, = torch.autograd.grad(autograd.head_norm_rotary(split(packed)[0], None, w)[0].sum(), (w,))
    assert only.shape == (d,)


def test_graph_replays(pkg):
    B, N, H, d = 2, 300, 4, 128
    Xq, Xk, wq, wk, dQ, dK, positions, inv_freq, sections = _case(B, N, H, H, d, "bf16", 1, torch.int64, 13)
    kw = dict(positions=positions, inv_freq=inv_freq)
    call = lambda: (*pkg.sphattn_head_norm_rotary_fwd(Xq, Xk, wq, wk, **kw), *pkg.sphattn_head_norm_rotary_bwd(Xq, Xk, wq, wk, dQ, dK, **kw))
    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = call()
    for i in range(3):
        with torch.no_grad():
            Xq.mul_(1.1)
            dK.add_(0.25)
            positions.add_(17)
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(out, call()):
            assert torch.equal(a, b), i

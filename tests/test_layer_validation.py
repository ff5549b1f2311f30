"""What the entry points of include/sphattn_layer.h refuse, without a GPU: the C ABI with addresses that are never followed, and the
binding's own checks."""
import ctypes
import os

import pytest
import torch

import paper_2505_09326_amd as pkg
from paper_2505_09326_amd import autograd


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(pkg.LIB_PATH):
        pkg.build_library()
    return pkg.load_library()


P = ctypes.c_void_p
WS = 0x700000000


def _view(data, batch, token, head):
    return ctypes.byref(pkg._Heads(data, batch, token, head))


def _rotary(positions=0x1000, id_bytes=8, axis=0, batch=10, inv_freq=0x8000, axes=1, sections=(32, 0, 0), interleaved=0):
    return ctypes.byref(pkg._Rotary(positions, id_bytes, axis, batch, inv_freq, axes, (ctypes.c_int * 3)(*sections), interleaved))


def test_head_norm_rotary_errors(lib):
    B, N, H, d = 2, 10, 4, 64
    by_token, by_head = (N * H * d, H * d, d), (H * N * d, d, N * d)

    def fwd(Xq=0x1000000, Xk=0x2000000, wq=0x9000, wk=0xa000, Q=0x3000000, K=0x4000000, rotary=_rotary(), B=B, N=N, Hq=H, Hk=H, d=d, norm=1, eps=1e-6,
            dtype=1, qs=by_head, xs=by_token):
        return lib.sphattn_head_norm_rotary_fwd(Xq and _view(Xq, *xs), Xk and _view(Xk, *by_token), P(wq), P(wk), Q and _view(Q, *qs), K and _view(K, *by_head),
                                                rotary, B, N, Hq, Hk, d, norm, eps, dtype, None)
    assert fwd(Xq=None) == -1 and fwd(Xk=None) == -1 and fwd(Q=None) == -1 and fwd(K=None) == -1 and fwd(rotary=_rotary(inv_freq=None)) == -1
    assert fwd(B=-1) == -2 and fwd(N=-1) == -2 and fwd(Hq=0) == -2 and fwd(Hk=-1) == -2 and fwd(Hq=65535, Hk=2) == -2 and fwd(B=65536, N=65536) == -2
    assert fwd(xs=(-1, H * d, d)) == -2 and fwd(xs=(2 ** 60, H * d, d)) == -2
    assert fwd(rotary=_rotary(axes=0)) == -2 and fwd(rotary=_rotary(axes=4)) == -2 and fwd(rotary=_rotary(sections=(31, 0, 0))) == -2
    assert fwd(rotary=_rotary(sections=(33, -1, 0), axes=2)) == -2 and fwd(rotary=_rotary(axis=-1)) == -2 and fwd(rotary=_rotary(batch=-1)) == -2
    assert fwd(d=32) == -3 and fwd(d=96) == -3
    assert fwd(dtype=2) == -4 and fwd(dtype=7) == -4 and fwd(rotary=_rotary(id_bytes=2)) == -4
    assert fwd(Xq=0x1000001) == -5 and fwd(wq=0x9001) == -5 and fwd(Q=0x3000001) == -5 and fwd(rotary=_rotary(positions=0x1004)) == -5
    assert fwd(rotary=_rotary(inv_freq=0x8002)) == -5 and fwd(Xq=0x1000002, dtype=0) == -5
    assert fwd(norm=2) == -11 and fwd(eps=-1.0) == -11 and fwd(eps=float("nan")) == -11 and fwd(eps=float("inf")) == -11
    # outputs over inputs, and outputs whose rows share places
    assert fwd(Q=0x1000000) == -7 and fwd(K=0x2000000 + 64) == -7 and fwd(Q=0x9000 - 64) == -7 and fwd(K=0x1000) == -7 and fwd(Q=0x8000) == -7
    assert fwd(qs=(0, d, N * d)) == -7 and fwd(qs=(H * N * d, d - 1, N * d)) == -7 and fwd(qs=(H * N * d, d, d)) == -7
    assert fwd(B=0) == 0 and fwd(N=0) == 0

    assert lib.sphattn_head_norm_rotary_bwd_workspace_bytes(32) == 0
    need = lib.sphattn_head_norm_rotary_bwd_workspace_bytes(d)
    assert need > 0

    def bwd(Xq=0x1000000, dQ=0x3000000, dK=0x4000000, dXq=0x5000000, dXk=0x6000000, dwq=0xb000, dwk=0xc000, ws=WS, size=need, Hk=H, xs=by_token):
        return lib.sphattn_head_norm_rotary_bwd(Xq and _view(Xq, *by_token), _view(0x2000000, *by_token), P(0x9000), P(0xa000), dQ and _view(dQ, *by_head),
                                                dK and _view(dK, *by_head), dXq and _view(dXq, *xs), dXk and _view(dXk, *by_token), P(dwq), P(dwk),
                                                _rotary(), B, N, H, Hk, d, 1, 1e-6, 1, P(ws), size, None)
    assert bwd(Xq=None) == -1 and bwd(dQ=None) == -1 and bwd(dK=None) == -1 and bwd(dXq=None, dXk=None, dwq=None, dwk=None) == -1
    assert bwd(dwq=0xb001) == -5 and bwd(dXq=0x5000001) == -5
    assert bwd(ws=0) == -9 and bwd(ws=WS + 8) == -9 and bwd(size=need - 1) == -9
    assert bwd(dXq=0x1000000) == -7 and bwd(dXq=0x3000000) == -7 and bwd(dXk=WS) == -7 and bwd(dwq=0xc000) == -7 and bwd(dwq=0x9000) == -7
    assert bwd(xs=(N * H * d, 0, d)) == -7


def test_head_norm_rotary_binding_checks():
    x, w, at, f = torch.zeros(2, 5, 3, 64), torch.ones(64), torch.zeros((2, 5), dtype=torch.int64), torch.ones(32)
    call = pkg.sphattn_head_norm_rotary_fwd
    for bad in (lambda: call(x), lambda: call(x[0]), lambda: call(x.double()), lambda: call(x, x.half()), lambda: call(x, x[:1]), lambda: call(x, x[..., :32]),
                lambda: call(x, None, w[:32]), lambda: call(x, None, w.half()), lambda: call(x, None, None, w), lambda: call(x, x[:, :, :0]),
                lambda: call(x.transpose(2, 3).contiguous().transpose(2, 3)), lambda: call(x, positions=at), lambda: call(x, inv_freq=f),
                lambda: call(x, positions=at.float(), inv_freq=f), lambda: call(x, positions=at[:, :4], inv_freq=f), lambda: call(x, positions=at, inv_freq=f[:16]),
                lambda: call(x, positions=at, inv_freq=f.double()), lambda: call(x, positions=at, inv_freq=f, sections=[16, 16]),
                lambda: call(x, positions=at.expand(2, 2, 5), inv_freq=f), lambda: call(x, positions=at.expand(2, 2, 5), inv_freq=f, sections=[33, -1]),
                lambda: call(x, positions=at.expand(4, 2, 5), inv_freq=f, sections=[8, 8, 8, 8]), lambda: call(x, positions=at.t().contiguous().t(), inv_freq=f),
                lambda: call(x, eps=-1.0), lambda: call(x, eps=float("nan")), lambda: call(x, Q=torch.zeros(2, 5, 3, 64)), lambda: call(x, K=x),
                lambda: call(x, stream=0)):
        with pytest.raises(ValueError):
            bad()
    back, g = pkg.sphattn_head_norm_rotary_bwd, torch.zeros(2, 3, 5, 64)
    for bad in (lambda: back(x, None, None, None, g, None), lambda: back(x, None, w, None, g, g), lambda: back(x, x, w, w, g, None), lambda: back(x, None, w, None, x, None),
                lambda: back(x, None, w, None, g, None, want_dX=(False, True), want_dw=(False, True)), lambda: back(x, None, w, None, g, None, dXq=g),
                lambda: back(x, None, w, None, g, None, stream=0)):
        with pytest.raises(ValueError):
            bad()
    with pytest.raises(ValueError):
        autograd.head_norm_rotary(x, x)                        # not on a GPU


def test_gated_ffn_errors(lib):
    T, D, F = 100, 64, 96
    size, back_size = lib.sphattn_gated_ffn_workspace_bytes, lib.sphattn_gated_ffn_bwd_workspace_bytes
    for f in (size, back_size):
        assert f(T, D, F, 1) > 0 and f(T, D, F, 0) > f(T, D, F, 1)
        assert f(-1, D, F, 1) == f(T, 0, F, 1) == f(T, D, 0, 1) == f(T, D, F, 2) == f(2 ** 20 + 1, D, F, 1) == f(2 ** 20, D, 2 ** 18, 1) == f(T, 65537, F, 1) == 0
    assert size(64, D, F, 0) == 0 and back_size(64, D, F, 1) > 0 and back_size(T, D, F, 3) > back_size(T, D, F, 1)
    need = size(T, D, F, 1)

    def fwd(X=0x1000000, Wg=0x2000000, Wu=0x3000000, H=0x4000000, T=T, D=D, F=F, gate=0, dtype=1, ws=WS, size=need):
        return lib.sphattn_gated_ffn_fwd(P(X), P(Wg), P(Wu), P(H), T, D, F, gate, dtype, P(ws), size, None)
    assert fwd(X=0) == -1 and fwd(Wg=0) == -1 and fwd(Wu=0) == -1 and fwd(H=0) == -1
    assert fwd(T=-1) == -2 and fwd(D=0) == -2 and fwd(F=2 ** 18 + 1) == -2 and fwd(T=2 ** 20, F=2 ** 17) == -2
    assert fwd(dtype=2) == -4 and fwd(X=0x1000001) == -5 and fwd(H=0x4000002, dtype=0) == -5 and fwd(gate=3) == -11 and fwd(gate=-1) == -11
    assert fwd(ws=0) == -9 and fwd(ws=WS + 8) == -9 and fwd(size=need - 1) == -9
    assert fwd(H=0x1000000) == -7 and fwd(H=0x2000000 + 64) == -7 and fwd(H=WS) == -7 and fwd(X=WS + 16) == -7
    assert fwd(T=0, X=0, H=0, ws=0, size=0) == 0
    need = back_size(T, D, F, 1)

    def bwd(X=0x1000000, Wg=0x2000000, Wu=0x3000000, dH=0x4000000, dX=0x5000000, dWg=0x6000000, dWu=0x7000000, gate=0, dtype=1, ws=WS, size=need, T=T):
        return lib.sphattn_gated_ffn_bwd(P(X), P(Wg), P(Wu), P(dH), P(dX), P(dWg), P(dWu), T, D, F, gate, dtype, P(ws), size, None)
    assert bwd(X=0) == -1 and bwd(dH=0) == -1 and bwd(dX=0, dWg=0, dWu=0) == -1
    assert bwd(T=-1) == -2 and bwd(dtype=7) == -4 and bwd(dWu=0x7000001) == -5 and bwd(gate=9) == -11
    assert bwd(ws=0) == -9 and bwd(size=need - 1) == -9
    assert bwd(dX=0x1000000) == -7 and bwd(dWg=0x7000000) == -7 and bwd(dWu=0x4000000) == -7 and bwd(dX=WS) == -7 and bwd(dWg=0x2000000 + 2) == -7


def test_gated_ffn_binding_checks():
    X, W, H = torch.zeros(10, 8), torch.zeros(12, 8), torch.zeros(10, 12)
    fwd, bwd = pkg.sphattn_gated_ffn_fwd, pkg.sphattn_gated_ffn_bwd
    for bad in (lambda: fwd(X, W, W), lambda: fwd(X[0], W, W), lambda: fwd(X, W[:, :4], W), lambda: fwd(X, W, W.half()), lambda: fwd(X.double(), W, W),
                lambda: fwd(X.t().contiguous().t(), W, W), lambda: fwd(X, W, W, stream=0), lambda: bwd(X, W, W, H[:9]), lambda: bwd(X, W, W, H.half()),
                lambda: bwd(X, W, W, H, want_dX=False, want_dWg=False, want_dWu=False), lambda: bwd(X, W, W, H, stream=0)):
        with pytest.raises(ValueError):
            bad()
    with pytest.raises(KeyError):
        fwd(X, W, W, "tanh")
    with pytest.raises(TypeError):
        autograd.gated_feed_forward(X, W.half(), W)


def test_distillation_errors(lib):
    T, V, D, K = 100, 500, 64, 20
    sizes = [lib.sphattn_vocab_distill_workspace_bytes, lib.sphattn_vocab_distill_bwd_workspace_bytes]
    for size in sizes:
        assert size(T, V, D, K, 1) > 0 and size(T, V, D, K, 0) > size(T, V, D, K, 1)
        assert size(-1, V, D, K, 1) == size(T, 0, D, K, 1) == size(T, V, D, 0, 1) == size(T, V, D, 1025, 1) == size(T, V, D, K, 2) == size(T, 2 ** 24 + 1, D, K, 1) == 0
    for T2 in (1, 2 ** 20):                        # no size of the ranges overflows on the way
        for V2 in (1, 50003, 2 ** 24):
            for K2 in (1, 1024):
                assert sizes[0](T2, V2, D, K2, 1) > 2 * (T2 + V2) * D + 12 * T2 * K2 and sizes[1](T2, V2, D, K2, 1) > 8 * T2 * K2
                assert sizes[0](T2, V2, D, K2, 1) < 4 * (T2 + V2) * D + 16 * T2 * K2 + T2 * V2 // 8 + (1 << 30)
    need = sizes[0](T, V, D, K, 1)

    def fwd(X=0x1000000, W=0x2000000, ids=0x3000000, id_bytes=8, teacher=0x3800000, losses=0x4000000, lse=0x4100000, kept=0x4200000, mean=0x4300000, T=T, V=V, K=K,
            scale=1.0, tau=1.0, reduction=2, dtype=1, ws=WS, size=need):
        return lib.sphattn_vocab_distill_fwd(P(X), P(W), P(ids), id_bytes, P(teacher), P(losses), P(lse), P(kept), P(mean), T, V, D, K, scale, tau, reduction,
                                             dtype, P(ws), size, None)
    assert fwd(X=0) == -1 and fwd(W=0) == -1 and fwd(ids=0) == -1 and fwd(teacher=0) == -1 and fwd(losses=0) == -1 and fwd(lse=0) == -1
    assert fwd(T=-1) == -2 and fwd(V=0) == -2 and fwd(K=0) == -2 and fwd(K=1025) == -2
    assert fwd(dtype=2) == -4 and fwd(id_bytes=2) == -4 and fwd(teacher=0x3800002) == -5 and fwd(kept=0x4200002) == -5 and fwd(ids=0x3000004) == -5
    assert fwd(scale=float("inf")) == -11 and fwd(reduction=3) == -11
    for tau in (0.0, -1.0, float("nan"), float("inf"), 2.0 ** -21, 2.0 ** 21):
        assert fwd(tau=tau) == -11
    assert fwd(scale=3e38, tau=2.0 ** -20) == -11
    assert fwd(ws=0) == -9 and fwd(ws=WS + 4) == -9 and fwd(size=need - 1) == -9
    assert fwd(kept=0x3800000) == -7 and fwd(lse=0x4000000) == -7 and fwd(losses=0x3000000) == -7 and fwd(W=WS) == -7 and fwd(kept=WS + need - 4) == -7
    need = sizes[1](T, V, D, K, 1)

    def bwd(X=0x1000000, lse=0x4100000, kept=0x4200000, dloss=0x4300000, dX=0x5000000, dW=0x6000000, tau=1.0, reduction=2, ws=WS, size=need, teacher=0x3800000):
        return lib.sphattn_vocab_distill_bwd(P(X), P(0x2000000), P(0x3000000), 8, P(teacher), P(lse), P(kept), P(dloss), P(dX), P(dW), T, V, D, K, 1.0, tau,
                                             reduction, 1, P(ws), size, None)
    assert bwd(lse=0) == -1 and bwd(kept=0) == -1 and bwd(dloss=0) == -1 and bwd(dX=0, dW=0) == -1 and bwd(teacher=0) == -1
    assert bwd(dX=0x5000001) == -5 and bwd(tau=0.0) == -11 and bwd(reduction=-1) == -11 and bwd(ws=0) == -9 and bwd(size=need - 1) == -9
    assert bwd(dX=0x1000000) == -7 and bwd(dW=0x2000000 + 64) == -7 and bwd(dW=0x4200000) == -7 and bwd(dX=0x6000000) == -7


def test_distillation_binding_checks():
    X, W, ids, teacher, one = torch.zeros(6, 8), torch.zeros(12, 8), torch.zeros((6, 3), dtype=torch.int64), torch.zeros(6, 3), torch.ones(6)
    fwd, bwd = pkg.sphattn_vocab_distill_fwd, pkg.sphattn_vocab_distill_bwd
    for bad in (lambda: fwd(X, W, ids, teacher), lambda: fwd(X, W, ids[:5], teacher), lambda: fwd(X, W, ids, teacher[:, :2]), lambda: fwd(X, W, ids.float(), teacher),
                lambda: fwd(X, W, ids, teacher.double()), lambda: fwd(X, W.half(), ids, teacher), lambda: fwd(X, W, ids[0], teacher), lambda: fwd(X, W[:, :4], ids, teacher),
                lambda: fwd(X, W, ids, teacher, float("nan")), lambda: fwd(X, W, ids, teacher, 1.0, 0.0), lambda: fwd(X, W, ids, teacher, 1.0, float("nan")),
                lambda: fwd(X, W, ids, teacher, stream=0), lambda: fwd(X, W, ids.t().contiguous().t(), teacher), lambda: bwd(X, W, ids, teacher, one, teacher, one),
                lambda: bwd(X, W, ids, teacher, one, teacher[:3], one), lambda: bwd(X, W, ids, teacher, one, teacher, one[:2]),
                lambda: bwd(X, W, ids, teacher, one, teacher, one, reduction="mean"), lambda: bwd(X, W, ids, teacher, one, teacher, one, want_dX=False, want_dW=False),
                lambda: bwd(X, W, ids, teacher, one, teacher, one, stream=0), lambda: autograd.vocab_distillation(X, W, ids[:5], teacher[:5]),
                lambda: autograd.vocab_distillation(X, W, ids, teacher[:5]), lambda: autograd.vocab_distillation(X, W, ids, teacher, temperature=-1.0)):
        with pytest.raises(ValueError):
            bad()
    with pytest.raises(KeyError):
        fwd(X, W, ids, teacher, reduction="most")

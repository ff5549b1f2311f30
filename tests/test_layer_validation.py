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

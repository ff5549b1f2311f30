"""What the entry points of include/sphattn_train.h refuse, without a GPU: the C ABI with addresses that are never followed, and the
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


def test_embedding_errors(lib):
    def fwd(tokens=0x1000, id_bytes=8, table=0x2000000, mult=None, O=0x6000000, T=100, V=50, D=64, dtype=1):
        return lib.sphattn_embed_fwd(P(tokens), id_bytes, P(table), P(mult), P(O), T, V, D, 1.0, dtype, None)
    assert fwd(tokens=0) == -1 and fwd(table=0) == -1 and fwd(O=0) == -1
    assert fwd(T=-1) == -2 and fwd(V=0) == -2 and fwd(D=0) == -2 and fwd(D=65537) == -2 and fwd(V=2 ** 30 + 1) == -2
    assert fwd(dtype=2) == -4 and fwd(dtype=9) == -4 and fwd(id_bytes=2) == -4
    assert fwd(table=0x2000001) == -5 and fwd(tokens=0x1004) == -5 and fwd(mult=0x5002) == -5 and fwd(O=0x6000002, dtype=0) == -5
    assert fwd(O=0x2000000) == -7 and fwd(O=0x1000 + 792) == -7 and fwd(mult=0x6000000 + 12796) == -7
    assert fwd(T=0, tokens=0, O=0) == 0

    need = lib.sphattn_embed_bwd_workspace_bytes(100, 50, 64)
    assert need > 0 and lib.sphattn_embed_bwd_workspace_bytes(-1, 50, 64) == 0 and lib.sphattn_embed_bwd_workspace_bytes(1, 0, 64) == 0

    def bwd(tokens=0x1000, mult=None, dO=0x2000000, dtable=0x6000000, ws=WS, size=need, D=64, dtype=1):
        return lib.sphattn_embed_bwd(P(tokens), 8, P(mult), P(dO), P(dtable), 100, 50, D, 1.0, dtype, P(ws), size, None)
    assert bwd(dO=0) == -1 and bwd(dtable=0) == -1 and bwd(tokens=0) == -1
    assert bwd(D=-3) == -2 and bwd(dtype=4) == -4 and bwd(dO=0x2000001) == -5
    assert bwd(ws=0) == -9 and bwd(ws=WS + 8) == -9 and bwd(size=need - 1) == -9
    assert bwd(dtable=0x2000000) == -7 and bwd(dO=WS + 64) == -7 and bwd(dtable=WS) == -7


def test_vocabulary_loss_errors(lib):
    T, V, D = 100, 500, 64
    sizes = [lib.sphattn_vocab_loss_workspace_bytes, lib.sphattn_vocab_loss_bwd_workspace_bytes]
    for size in sizes:
        assert size(T, V, D, 1) > 0 and size(T, V, D, 0) > size(T, V, D, 1)
        assert size(-1, V, D, 1) == size(T, 0, D, 1) == size(T, V, D, 2) == size(2 ** 20 + 1, V, D, 1) == 0
    need = sizes[0](T, V, D, 1)

    def fwd(X=0x1000000, W=0x2000000, targets=0x3000000, id_bytes=8, losses=0x4000000, lse=0x4100000, mean=0x4200000, T=T, V=V, D=D, scale=1.0,
            reduction=2, dtype=1, ws=WS, size=need):
        return lib.sphattn_vocab_loss_fwd(P(X), P(W), P(targets), id_bytes, P(losses), P(lse), P(mean), T, V, D, scale, reduction, 1, dtype,
                                          P(ws), size, None)
    assert fwd(X=0) == -1 and fwd(W=0) == -1 and fwd(targets=0) == -1 and fwd(losses=0) == -1
    assert fwd(T=-1) == -2 and fwd(V=0) == -2 and fwd(V=2 ** 24 + 1) == -2 and fwd(D=0) == -2
    assert fwd(dtype=2) == -4 and fwd(id_bytes=1) == -4
    assert fwd(X=0x1000001) == -5 and fwd(lse=0x4100002) == -5 and fwd(targets=0x3000004) == -5
    assert fwd(scale=float("nan")) == -11 and fwd(scale=float("inf")) == -11 and fwd(reduction=3) == -11 and fwd(reduction=-1) == -11
    assert fwd(ws=0) == -9 and fwd(size=need - 1) == -9 and fwd(ws=WS + 4) == -9
    assert fwd(lse=0x4000000) == -7 and fwd(mean=0x4000000 + 396) == -7 and fwd(losses=0x1000000 + 128) == -7 and fwd(W=WS) == -7

    need = sizes[1](T, V, D, 1)

    def bwd(X=0x1000000, W=0x2000000, targets=0x3000000, lse=0x4100000, dloss=0x4200000, dX=0x5000000, dW=0x6000000, reduction=2, dtype=1, ws=WS,
            size=need, scale=1.0):
        return lib.sphattn_vocab_loss_bwd(P(X), P(W), P(targets), 8, P(lse), P(dloss), P(dX), P(dW), T, V, D, scale, reduction, dtype, P(ws), size, None)
    assert bwd(lse=0) == -1 and bwd(dloss=0) == -1 and bwd(dX=0, dW=0) == -1
    assert bwd(dX=0x5000001) == -5 and bwd(dloss=0x4200002) == -5
    assert bwd(reduction=7) == -11 and bwd(scale=float("nan")) == -11
    assert bwd(ws=0) == -9 and bwd(size=need - 1) == -9
    assert bwd(dX=0x1000000) == -7 and bwd(dW=0x2000000 + 64) == -7 and bwd(dX=0x6000000) == -7 and bwd(dloss=WS) == -7


def test_workspaces_hold_what_their_sizes_say(lib):
    """No size of the ranges that the calls take overflows on the way to its workspace."""
    for T in (0, 1, 4097, 2 ** 20):
        for V in (1, 50003, 2 ** 24):
            for D in (1, 515, 65536):
                for dtype, parts in ((0, 2), (1, 1), (3, 1)):
                    at_least = 2 * parts * (T + V) * D
                    assert lib.sphattn_vocab_loss_workspace_bytes(T, V, D, dtype) > at_least
                    assert lib.sphattn_vocab_loss_bwd_workspace_bytes(T, V, D, dtype) > at_least + 4 * T * D
    assert lib.sphattn_embed_bwd_workspace_bytes(2 ** 31 - 1, 2 ** 30, 65536) > 2 ** 33


def test_clip_errors(lib):
    need = lib.sphattn_clip_grads_workspace_bytes(2)
    assert need > 0 and lib.sphattn_clip_grads_workspace_bytes(-1) == 0 and lib.sphattn_clip_grads_workspace_bytes(0) > 0
    assert lib.sphattn_clip_grads_workspace_bytes(121) == 2 * need

    def call(a=0x1000, b=0x2000000, oa=0x3000000, ob=0x4000000, sizes=(100, 200), types=(0, 1), n=2, limit=1.0, norm=0x5000000, ws=WS, size=need, none=False):
        ptr = ctypes.c_void_p * 2
        return lib.sphattn_clip_grads(None if none else ptr(a, b), ptr(oa, ob), (ctypes.c_longlong * 2)(*sizes), (ctypes.c_int * 2)(*types), n, limit,
                                      P(norm), P(ws), size, None)
    assert call(n=-1) == -2 and call(sizes=(100, -1)) == -2
    assert call(none=True) == -1 and call(norm=0) == -1 and call(b=None) == -1 and call(ob=None) == -1
    assert call(types=(0, 2)) == -4
    assert call(a=0x1002) == -5 and call(norm=0x5000001) == -5
    assert call(limit=-1.0) == -11 and call(limit=float("nan")) == -11
    assert call(ws=0) == -9 and call(size=need - 1) == -9
    assert call(oa=0x1000 + 4) == -7 and call(ob=0x5000000) == -7 and call(a=WS) == -7 and call(norm=WS) == -7


def _expect(text, call):
    with pytest.raises(ValueError, match=text):
        call()


def test_binding_embedding():
    tokens, table, dO = torch.zeros(5, dtype=torch.int64), torch.zeros(7, 8), torch.zeros(5, 8)
    _expect("device tensor", lambda: pkg.sphattn_embed_fwd(tokens, table))
    _expect("one-dimensional", lambda: pkg.sphattn_embed_fwd(tokens.view(1, 5), table))
    _expect("dtype", lambda: pkg.sphattn_embed_fwd(tokens.float(), table))
    _expect("dtype", lambda: pkg.sphattn_embed_fwd(tokens, table.double()))
    _expect("contiguous", lambda: pkg.sphattn_embed_fwd(tokens, table.t()))
    _expect("shape", lambda: pkg.sphattn_embed_fwd(tokens, table, mult=torch.ones(4)))
    _expect("dtype", lambda: pkg.sphattn_embed_fwd(tokens, table, mult=torch.ones(5).double()))
    _expect("shape", lambda: pkg.sphattn_embed_fwd(tokens, table, O=torch.zeros(5, 9)))
    _expect("O is required", lambda: pkg.sphattn_embed_fwd(tokens, table, stream=0))
    _expect("shape", lambda: pkg.sphattn_embed_bwd(tokens, torch.zeros(6, 8), 7))
    _expect("device tensor", lambda: pkg.sphattn_embed_bwd(tokens, dO, 7))
    _expect("workspace is required", lambda: pkg.sphattn_embed_bwd(tokens, dO, 7, dtable=table, stream=0))
    _expect("shape", lambda: autograd.token_embedding(tokens, table, mult=torch.ones(1, 5)))


def test_binding_vocabulary_loss():
    X, W, y = torch.zeros(5, 8), torch.zeros(7, 8), torch.zeros(5, dtype=torch.int64)
    lse, one = torch.zeros(5), torch.ones(())
    _expect("device tensor", lambda: pkg.sphattn_vocab_loss_fwd(X, W, y))
    _expect("two-dimensional", lambda: pkg.sphattn_vocab_loss_fwd(X[0], W, y))
    _expect("shape", lambda: pkg.sphattn_vocab_loss_fwd(X, torch.zeros(7, 9), y))
    _expect("dtype", lambda: pkg.sphattn_vocab_loss_fwd(X, W.bfloat16(), y))
    _expect("dtype", lambda: pkg.sphattn_vocab_loss_fwd(X.double(), W.double(), y))
    _expect("shape", lambda: pkg.sphattn_vocab_loss_fwd(X, W, y[:4]))
    _expect("dtype", lambda: pkg.sphattn_vocab_loss_fwd(X, W, y.float()))
    _expect("finite", lambda: pkg.sphattn_vocab_loss_fwd(X, W, y, scale=float("nan")))
    _expect("contiguous", lambda: pkg.sphattn_vocab_loss_fwd(torch.zeros(8, 5).t(), W, y))
    _expect("lse is required", lambda: pkg.sphattn_vocab_loss_fwd(X, W, y, losses=lse, stream=0))
    with pytest.raises(KeyError):
        pkg.sphattn_vocab_loss_fwd(X, W, y, reduction="median")
    _expect("lse is required", lambda: pkg.sphattn_vocab_loss_bwd(X, W, y, None, one, reduction="mean"))
    _expect("shape", lambda: pkg.sphattn_vocab_loss_bwd(X, W, y, lse, one))
    _expect("shape", lambda: pkg.sphattn_vocab_loss_bwd(X, W, y, lse, lse, reduction="sum"))
    _expect("neither", lambda: pkg.sphattn_vocab_loss_bwd(X, W, y, lse, one, reduction="sum", want_dX=False, want_dW=False))
    _expect("device tensor", lambda: pkg.sphattn_vocab_loss_bwd(X, W, y, lse, one, reduction="sum"))
    _expect("shape of X's rows", lambda: autograd.vocab_cross_entropy(X.view(1, 5, 8), W, y))
    with pytest.raises(TypeError):
        autograd.vocab_cross_entropy(X, W.half(), y)


def test_binding_clip():
    x = torch.zeros(4)
    _expect("on a GPU|a GPU", lambda: pkg.sphattn_clip_grads([x], 1.0))
    _expect("max_norm", lambda: pkg.sphattn_clip_grads([x], -1.0))
    _expect("max_norm", lambda: pkg.sphattn_clip_grads([x], float("nan")))
    _expect("1 tensors", lambda: pkg.sphattn_clip_grads([x], 1.0, out=[]))
    _expect("no gradients", lambda: pkg.sphattn_clip_grads([], 1.0))


def test_dense_in_memory():
    t = torch.zeros(4, 6, 5)
    assert pkg._dense(t) and pkg._dense(t.permute(2, 0, 1)) and pkg._dense(t[:1]) and pkg._dense(torch.zeros(())) and pkg._dense(t[:, :0])
    assert not pkg._dense(t[:, :3]) and not pkg._dense(t[:, 0]) and not pkg._dense(torch.zeros(1, 3).expand(4, 3))

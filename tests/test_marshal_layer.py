"""_marshal in front of heads, gated feed-forward and distillation: the Python path's results bit for bit, what is not right left to that path."""
import os

import pytest
import torch

import paper_2505_09326_amd as pkg
from paper_2505_09326_amd import autograd
from paper_2505_09326_amd._build import MARSHAL_PATH, build_marshal

DEV = "cuda:0"


def test_what_is_not_right_is_left_to_python():
    if not os.path.exists(MARSHAL_PATH):
        build_marshal()
    fast = pkg._bound_marshal(pkg.load_library())
    x, w, f, at = torch.zeros(2, 5, 3, 64), torch.ones(64), torch.ones(32), torch.zeros(5, dtype=torch.int64)
    assert fast.heads_forward(x, x, w, w, at, f, None, False, True, 1e-6, None, None, True) is None        # not on a device
    assert fast.heads_forward(x, [x], w, w, at, f, None, False, True, 1e-6, None, None, True) is None
    assert fast.heads_forward(x, None, None, None, None, None, (32,), False, True, 1e-6, None, None, False) is None
    assert fast.heads_forward(x, None, None, None, None, None, None, False, True, -1.0, None, None, False) is None
    assert fast.ffn_forward(x[0, 0], w, w, 0, False) is None and fast.ffn_forward(None, w, w, 0, True) is None
    ids = torch.zeros((3, 4), dtype=torch.int64)
    assert fast.distill_forward(x[0, 0], x[0, 0], ids, torch.zeros(3, 4), 1.0, 1.0, 0, False, False) is None
    with pytest.raises(TypeError):
        fast.heads_forward(x)
    with pytest.raises(TypeError):
        fast.ffn_forward(x, w, w, "silu", True)
    with pytest.raises(TypeError):
        fast.distill_forward(x, x, ids, x, "1", 1.0, 0, False, True)


def _same(a, b):
    assert len(a) == len(b)
    for x, y in zip(a, b):
        assert (x is None) == (y is None)
        if x is not None:
            same = torch.equal(x, y)
            assert x.dtype == y.dtype and x.stride() == y.stride() and x.requires_grad == y.requires_grad and same


def _calls(dtype):
    g = torch.Generator(device=DEV).manual_seed(1)
    r = lambda *s: torch.randn(s, generator=g, device=DEV).to(dtype)
    leaf = lambda t: t.detach().clone().requires_grad_(True)
    packed = leaf(r(2, 7, 6 * 64))
    wq, wk, f = leaf(r(64)), leaf(r(64)), torch.rand(32, generator=g, device=DEV)
    q = lambda: packed[..., :256].view(2, 7, 4, 64)
    k = lambda: packed[..., 256:].view(2, 7, 2, 64)
    at1, at2, at3 = torch.arange(7, device=DEV), torch.arange(14, device=DEV, dtype=torch.int32).view(2, 7), torch.arange(42, device=DEV).view(3, 2, 7)
    X, Wg, Wu = leaf(r(3, 30, 40)), leaf(r(50, 40)), leaf(r(50, 40))
    W = leaf(r(60, 40))
    ids, teacher = torch.randint(-1, 60, (3, 30, 5), generator=g, device=DEV), torch.randn((3, 30, 5), generator=g, device=DEV)
    flat = lambda t: t.detach().reshape(-1, t.shape[-1])
    cache = torch.zeros(2, 2, 20, 64, device=DEV, dtype=dtype)

    def grads(outs, leaves):
        outs = [o for o in outs if o is not None]
        return [o.detach() for o in outs] + list(torch.autograd.grad([o.float().square().sum() for o in outs], leaves))
    yield lambda: pkg.sphattn_head_norm_rotary_fwd(q().detach(), k().detach(), wq.detach(), None, at1, f)
    yield lambda: pkg.sphattn_head_norm_rotary_fwd(q().detach(), None, None, None, at3, f, [10, 2, 20], True, False)
    yield lambda: (*pkg.sphattn_head_norm_rotary_fwd(q().detach(), k().detach(), None, wk.detach(), at2, f, K=cache[:, :, 3:10]), cache.clone())
    yield lambda: pkg.sphattn_head_norm_rotary_fwd(q().detach(), k().detach(), eps=0.5)
    yield lambda: grads(autograd.head_norm_rotary(q(), k(), wq, wk, at2, f, None, True, True, 1e-3), (packed, wq, wk))
    yield lambda: grads(autograd.head_norm_rotary(q(), k(), wq, wk, at3, f, [10, 2, 20]), (packed, wk))
    yield lambda: grads(autograd.head_norm_rotary(q(), k(), wq, wk, norm=False), (packed, wq))
    yield lambda: grads(autograd.head_norm_rotary(q(), k(), wq.detach(), wk, at1, f), (packed,))
    yield lambda: grads(autograd.head_norm_rotary(q(), None, wq), (wq,))
    yield lambda: (pkg.sphattn_gated_ffn_fwd(flat(X), Wg.detach(), Wu.detach(), "relu"), pkg.sphattn_gated_ffn_fwd(flat(X)[:3], Wg.detach(), Wu.detach()))
    yield lambda: grads([autograd.gated_feed_forward(X, Wg, Wu, "gelu")], (X, Wg, Wu))
    yield lambda: grads([autograd.gated_feed_forward(X[0], Wg.detach(), Wu)], (Wu,))
    for reduction in ("none", "sum", "mean"):
        yield lambda: pkg.sphattn_vocab_distill_fwd(flat(X), W.detach(), flat(ids), flat(teacher), 0.5, 2.0, reduction)
        yield lambda: pkg.sphattn_vocab_distill_fwd(flat(X), W.detach(), flat(ids).int(), flat(teacher), reduction=reduction, keep=True)
        yield lambda: grads([autograd.vocab_distillation(X, W, ids, teacher, 0.5, 2.0, reduction)], (X, W))
    yield lambda: grads([autograd.vocab_distillation(X.detach(), W, ids, teacher)], (W,))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
def test_calls_equal_the_python_path(monkeypatch, dtype):
    fast = [c() for c in _calls(dtype)]
    used = []
    real = pkg._fast

    class Slow(pkg._PythonOnly):
        @staticmethod
        def heads_forward(*args):
            used.append("heads")
        @staticmethod
        def ffn_forward(*args):
            used.append("ffn")
        @staticmethod
        def distill_forward(*args):
            used.append("distill")
    with monkeypatch.context() as patch:
        patch.setattr(pkg, "_fast", Slow)
        slow = [c() for c in _calls(dtype)]
    assert pkg._fast is real and set(used) == {"heads", "ffn", "distill"}
    for a, b in zip(fast, slow):
        _same(a, b)


@pytest.mark.gpu
def test_it_was_not_python_that_did_them(monkeypatch):
    calls = list(_calls(torch.bfloat16))
    with monkeypatch.context() as patch:
        patch.setattr(pkg, "_projection", None)
        patch.setattr(pkg, "_gated", None)
        patch.setattr(pkg, "_taught", None)
        for i, c in enumerate(calls):
            if i != 8:                             # (one side alone with gradients is Python's)
                c()


@pytest.mark.gpu
def test_errors_are_the_bindings_own():
    X, W = torch.zeros(4, 8, device=DEV), torch.zeros(5, 8, device=DEV)
    q = torch.zeros(1, 2, 3, 32, device=DEV)
    with pytest.raises(pkg.SphattnError) as e:
        pkg.sphattn_head_norm_rotary_fwd(q)
    assert e.value.code == -3
    with pytest.raises(ValueError):
        pkg.sphattn_gated_ffn_fwd(X, W, W[:4])
    with pytest.raises(KeyError):
        pkg.sphattn_gated_ffn_fwd(X, W, W, "tanh")
    with pytest.raises(ValueError):
        pkg.sphattn_vocab_distill_fwd(X, W, torch.zeros((4, 2), device=DEV), torch.zeros((4, 2), device=DEV))
    with pytest.raises(pkg.SphattnError) as e:
        pkg.sphattn_vocab_distill_fwd(X, W, torch.zeros((4, 1025), dtype=torch.int64, device=DEV), torch.zeros((4, 1025), device=DEV))
    assert e.value.code == -2
    overlapping = torch.zeros(2, 3, 5, 64, device=DEV)
    with pytest.raises(pkg.SphattnError) as e:     # rows of the output in one place
        pkg.sphattn_head_norm_rotary_fwd(torch.zeros(2, 5, 3, 64, device=DEV), Q=overlapping[:, :1].expand(2, 3, 5, 64))
    assert e.value.code == -7
    x = torch.zeros(2, 5, 3, 64, device=DEV)
    with pytest.raises(pkg.SphattnError) as e:     # onto its input
        pkg.sphattn_head_norm_rotary_fwd(x, Q=x.transpose(1, 2))
    assert e.value.code == -7

"""_marshal in front of the calls of include/sphattn_train.h: the Python path's results bit for bit, what is not right left to that path, gradients
once and not twice."""
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
    tokens, table, X, lse = torch.zeros(5, dtype=torch.int64), torch.zeros(7, 8), torch.zeros(5, 8), torch.zeros(5)
    assert fast.embed_forward(tokens, table, None, 1.0, False) is None        # not on a device
    assert fast.embed_forward(tokens, None, None, 1.0, False) is None and fast.embed_forward(tokens, table, 3, 1.0, True) is None
    assert fast.embed_backward(tokens, X, 7, None, 1.0) is None
    assert fast.loss_forward(X, table, tokens, 1.0, 2, False, True) is None and fast.loss_forward(X, [table], tokens, 1.0, 2, False, False) is None
    assert fast.loss_backward(X, table, tokens, lse, torch.ones(()), 1.0, 2, True, True) is None
    assert fast.clip([X], [X], 1.0) is None and fast.clip((X,), (X,), 1.0) is None and fast.clip([], [], 1.0) is None and fast.clip([X], [X], -1.0) is None
    with pytest.raises(TypeError):
        fast.embed_forward(tokens, table)
    with pytest.raises(TypeError):
        fast.loss_forward(X, table, tokens, 1.0, "mean", False, True)


def _same(a, b):
    assert len(a) == len(b)
    for x, y in zip(a, b):
        assert (x is None) == (y is None)
        if x is not None:
            assert x.dtype == y.dtype and x.stride() == y.stride() and x.requires_grad == y.requires_grad and torch.equal(x, y)


def _inputs(dtype, ids, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    r = lambda *s: torch.randn(s, generator=g, device=DEV).to(dtype)
    tokens = torch.randint(-1, 50, (3, 20), generator=g, device=DEV).to(ids)
    return tokens, r(50, 40), torch.rand((3, 20), generator=g, device=DEV), r(3, 20, 40), torch.rand((3, 20), generator=g, device=DEV)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,ids", [(torch.float32, torch.int64), (torch.bfloat16, torch.int32), (torch.float16, torch.int64)])
def test_calls_equal_the_python_path(monkeypatch, dtype, ids):
    tokens, table, mult, X, dloss = _inputs(dtype, ids, 5)
    flat, rows = tokens.view(-1), X.view(60, 40)
    lse = pkg.sphattn_vocab_loss_fwd(rows, table, flat)[1]
    calls = [lambda: (pkg.sphattn_embed_fwd(flat, table, mult.view(-1), 0.3),), lambda: (pkg.sphattn_embed_bwd(flat, rows, 50, scale=2.0),),
             lambda: pkg.sphattn_vocab_loss_fwd(rows, table, flat, 0.5), lambda: pkg.sphattn_vocab_loss_fwd(rows, table, flat, reduction="sum", all_rows=False),
             lambda: pkg.sphattn_vocab_loss_bwd(rows, table, flat, lse, dloss.view(-1)), lambda: pkg.sphattn_vocab_loss_bwd(rows, table, flat, lse, dloss.view(-1), want_dW=False)]
    fast = [c() for c in calls]
    with monkeypatch.context() as patch:           # (it was not the Python path that did them)
        patch.setattr(pkg, "_ids", None)
        for c in calls:
            c()
    monkeypatch.setattr(pkg, "_fast", pkg._PythonOnly)
    for a, c in zip(fast, calls):
        _same(a, c())


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,ids", [(torch.float32, torch.int64), (torch.bfloat16, torch.int32), (torch.float16, torch.int64)])
@pytest.mark.parametrize("reduction", ["none", "sum", "mean"])
def test_training_step_equals_the_python_path(monkeypatch, dtype, ids, reduction):
    tokens, table, mult, X, dloss = _inputs(dtype, ids, 6)
    table.requires_grad_(True)
    X.requires_grad_(True)

    def step():
        out = autograd.token_embedding(tokens, table, mult, 0.3)
        loss = autograd.vocab_cross_entropy(X + out, table, tokens, 0.7, reduction)
        return [loss.detach(), out.detach(), *torch.autograd.grad(loss, (X, table), dloss if reduction == "none" else torch.tensor(3.0, device=DEV))]

    def frozen():                                  # one of the two at a time, and none
        a = autograd.vocab_cross_entropy(X.detach(), table, tokens, reduction="sum")
        b = autograd.vocab_cross_entropy(X, table.detach(), tokens, reduction="sum")
        c = autograd.vocab_cross_entropy(X.detach(), table.detach(), tokens, reduction=reduction)
        assert not c.requires_grad
        return [*torch.autograd.grad(a, (table,)), *torch.autograd.grad(b, (X,)), c]
    with monkeypatch.context() as patch:
        patch.setattr(pkg, "_ids", None)
        fast = step() + frozen()
    monkeypatch.setattr(pkg, "_fast", pkg._PythonOnly)
    _same(fast, step() + frozen())


@pytest.mark.gpu
def test_gradients_of_other_layouts(monkeypatch):
    """A gradient that is a broadcast value or transposed, inputs that are not contiguous, rows without a token."""
    tokens, table, mult, X, _ = _inputs(torch.float32, torch.int64, 7)
    X.requires_grad_(True)
    table.requires_grad_(True)
    calls = [lambda: torch.autograd.grad(autograd.token_embedding(tokens, table, mult).sum(), (table,)),
             lambda: torch.autograd.grad(autograd.token_embedding(tokens.t(), table, mult.t()), (table,), X.detach().transpose(0, 1)),
             lambda: torch.autograd.grad(autograd.vocab_cross_entropy(X.transpose(0, 1), table, tokens.t(), reduction="none").sum(), (X, table)),
             lambda: torch.autograd.grad(autograd.vocab_cross_entropy(X[:0], table, tokens[:0], reduction="sum"), (X, table))]
    got = [c() for c in calls]
    monkeypatch.setattr(pkg, "_fast", pkg._PythonOnly)
    for a, c in zip(got, calls):
        _same(a, c())


@pytest.mark.gpu
def test_without_multiplicities(monkeypatch):
    tokens, table, _, X, _ = _inputs(torch.bfloat16, torch.int64, 10)
    table.requires_grad_(True)

    def step():
        out = autograd.token_embedding(tokens, table, scale=0.3)
        return [out.detach(), *torch.autograd.grad(out, (table,), X)]
    with monkeypatch.context() as patch:
        patch.setattr(pkg, "_ids", None)
        fast = step()
    monkeypatch.setattr(pkg, "_fast", pkg._PythonOnly)
    _same(fast, step())


@pytest.mark.gpu
@pytest.mark.parametrize("python", [False, True])
def test_no_second_derivative(monkeypatch, python):
    if python:
        monkeypatch.setattr(pkg, "_fast", pkg._PythonOnly)
    tokens, table, mult, X, dloss = _inputs(torch.float32, torch.int64, 8)
    X.requires_grad_(True)
    table.requires_grad_(True)
    # (the second one's incoming gradient depends on X, as it does behind any further layer)
    for out, weight in ((autograd.token_embedding(tokens, table, mult), X), (autograd.vocab_cross_entropy(X, table, tokens, reduction="none"), X.sum(-1))):
        grad, = torch.autograd.grad((out * weight).sum(), (table,), create_graph=True)
        with pytest.raises(RuntimeError):
            grad.sum().backward()


@pytest.mark.gpu
@pytest.mark.parametrize("in_place", [False, True])
def test_clipping_equals_the_python_path(monkeypatch, in_place):
    g = torch.Generator(device=DEV).manual_seed(9)
    made = [torch.randn(s, generator=g, device=DEV).to(t) for s, t in (((70, 30), torch.float32), ((5,), torch.bfloat16), ((0,), torch.float32), ((9, 4), torch.float16))]
    made.append(torch.randn(6, 11, generator=g, device=DEV).t())

    def call():
        grads = [x.clone() for x in made]
        out = grads if in_place else [torch.empty_like(x) for x in grads]
        return [pkg.sphattn_clip_grads(grads, 0.5, out=None if in_place else out), *out]
    fast = call()
    with monkeypatch.context() as patch:
        patch.setattr(pkg, "_codes", None)
        call()
    monkeypatch.setattr(pkg, "_fast", pkg._PythonOnly)
    _same(fast, call())

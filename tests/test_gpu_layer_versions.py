"""Autograd is told of the caller's tensors that the layer's operators and the distillation write: a backward pass that saved one of them says so instead of using other values."""
import pytest
import torch

import paper_2505_09326_amd as pkg

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
bf16 = torch.bfloat16


def _randn(*shape):
    return torch.randn(shape, device=DEV)


def _calls():
    X, Wg, Wu, dH = _randn(5, 16).to(bf16), _randn(24, 16).to(bf16), _randn(24, 16).to(bf16), _randn(5, 24).to(bf16)
    ids, teacher = torch.randint(24, (5, 3), device=DEV), _randn(5, 3)
    heads, w, dQ = _randn(1, 4, 2, 64).to(bf16), _randn(64).to(bf16), _randn(1, 2, 4, 64).to(bf16)
    lse, kept, g = _randn(5), _randn(5, 3), _randn(5)
    f = lambda *shape: torch.empty(shape, device=DEV)
    h = lambda *shape: torch.empty(shape, device=DEV, dtype=bf16)
    return {
        "ffn": (lambda o: pkg.sphattn_gated_ffn_fwd(X, Wg, Wu, **o), {"H": h(5, 24)}),
        "ffn_bwd": (lambda o: pkg.sphattn_gated_ffn_bwd(X, Wg, Wu, dH, **o), {"dX": h(5, 16), "dWg": h(24, 16), "dWu": h(24, 16)}),
        "distill": (lambda o: pkg.sphattn_vocab_distill_fwd(X, Wg, ids, teacher, reduction="mean", **o), {"losses": f(5), "lse": f(5), "kept": f(5, 3), "mean": f()}),
        "distill_bwd": (lambda o: pkg.sphattn_vocab_distill_bwd(X, Wg, ids, teacher, lse, kept, g, **o), {"dX": h(5, 16), "dW": h(24, 16)}),
        "heads": (lambda o: pkg.sphattn_head_norm_rotary_fwd(heads, heads, w, w, **o), {"Q": h(1, 2, 4, 64), "K": h(1, 2, 4, 64)}),
        "heads_bwd": (lambda o: pkg.sphattn_head_norm_rotary_bwd(heads, heads, w, w, dQ, dQ, **o), {"dXq": h(1, 4, 2, 64), "dXk": h(1, 4, 2, 64), "dwq": h(64), "dwk": h(64)}),
    }


@pytest.mark.parametrize("python", [False, True])
@pytest.mark.parametrize("name", ["ffn", "ffn_bwd", "distill", "distill_bwd", "heads", "heads_bwd"])
def test_what_is_written_has_a_new_version(monkeypatch, name, python):
    if python:
        monkeypatch.setattr(pkg, "_fast", pkg._PythonOnly)
    call, out = _calls()[name]
    call(out)
    assert {k: t._version for k, t in out.items()} == {k: 1 for k in out}
    for k, t in out.items():
        weight = torch.ones_like(t).requires_grad_(True)
        y = (t * weight).sum()                                 # (saves t)
        call({k: t})
        with pytest.raises(RuntimeError, match="inplace operation"):
            y.backward()
    with torch.inference_mode():                               # (tensors of inference have no version)
        call, out = _calls()[name]
        call(out)

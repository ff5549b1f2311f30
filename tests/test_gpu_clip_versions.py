"""Autograd is told of tensors that clipping writes: a backward pass that saved one of them says so instead of using other values."""
import pytest
import torch

import paper_2505_09326_amd as pkg

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("python", [False, True])
@pytest.mark.parametrize("in_place", [False, True])
def test_what_was_saved_is_known_to_have_changed(monkeypatch, python, in_place):
    if python:
        monkeypatch.setattr(pkg, "_fast", pkg._PythonOnly)
    x = torch.full((100,), 3.0, device=DEV, requires_grad=True)
    y = x * 2
    z = (y * y).sum()                              # (saves y)
    grads, versions = [y.detach(), torch.ones(5, device=DEV)], [y._version, 0]
    if in_place:
        pkg.sphattn_clip_grads(grads, 1.0)
    else:
        pkg.sphattn_clip_grads([torch.ones_like(t) for t in grads], 1.0, out=grads)
    assert all(t._version > v for t, v in zip(grads, versions))
    with pytest.raises(RuntimeError, match="inplace operation"):
        z.backward()


@pytest.mark.parametrize("python", [False, True])
def test_what_is_only_read_keeps_its_version_and_inference_tensors_have_none(monkeypatch, python):
    if python:
        monkeypatch.setattr(pkg, "_fast", pkg._PythonOnly)
    x = torch.full((4,), 1.0, device=DEV)
    pkg.sphattn_clip_grads([x], 1.0, out=[torch.empty_like(x)])
    assert x._version == 0
    with torch.inference_mode():
        y = torch.full((4,), 1.0, device=DEV)
        assert float(pkg.sphattn_clip_grads([y], 1.0)) == 2.0
    assert abs(float(y[0]) - 0.5) < 1e-6

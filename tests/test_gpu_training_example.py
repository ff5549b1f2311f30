"""The example runs embedding, attention, vocabulary loss and clipping together: it starts at about log V and learns."""
import importlib.util
import math
import os

import pytest

pytestmark = pytest.mark.gpu
PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "..", "examples", "train_masked_genes.py")


def test_the_example_learns():
    spec = importlib.util.spec_from_file_location("train_masked_genes", PATH)
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    losses, norms = example.train(steps=80, batch=8, length=128, genes=500, types=5, heads=2)
    assert all(math.isfinite(x) for x in losses + norms)
    assert losses[0] > 0.8 * math.log(501) and sum(losses[-5:]) / 5 < losses[0] - 0.3

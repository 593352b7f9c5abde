"""The example that runs the operators together, at a small size with odd lengths."""
import importlib.util
import os

import pytest
import torch

pytestmark = pytest.mark.gpu
PATH = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "train_low_bits.py")


def load():
    spec = importlib.util.spec_from_file_location("train_low_bits", PATH)
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def test_it_learns_and_a_second_run_does_the_same():
    train = load().train
    runs = [train(steps=100, tokens=100, width=72, hidden=200, workers=3) for _ in range(2)]
    losses, (said, right), moments = runs[0]
    assert losses[-1] < losses[0] / 2
    assert said.shape == right.shape == (1, 72) and bool(torch.isfinite(said).all())
    assert all(bool(torch.isfinite(m).all()) and bool((m != 0).any()) for m in moments)
    assert losses == runs[1][0] and torch.equal(said, runs[1][1][0])
    assert all(torch.equal(a, b) for a, b in zip(moments, runs[1][2]))

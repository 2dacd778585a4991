"""The training example end to end: lookup, gradient, clipping, push and pull."""
import importlib.util
import os

import pytest

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_the_example_learns_and_compresses():
    spec = importlib.util.spec_from_file_location(
        "embedding_training", os.path.join(ROOT, "examples", "embedding_training.py"))
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    losses, share = example.train(steps=40, report=lambda text: print(text, flush=True))
    assert losses[-1] < 0.8 * losses[0]
    assert share < 1.6 / 8  # bytes a value: below the 1.6 bits of the quartic code

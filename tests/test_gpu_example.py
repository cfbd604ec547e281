"""The example that runs the 8-bit layers, the compressed step and the orthogonalised update together learns its task."""
import importlib.util
import os

import pytest

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_training_with_all_operators_learns():
    spec = importlib.util.spec_from_file_location("train_int8_orth", os.path.join(ROOT, "examples", "train_int8_orth.py"))
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    losses = example.train(steps=80)
    assert all(v == v and v < 100 for v in losses)
    assert sum(losses[-5:]) < 0.5 * sum(losses[:5])
    assert example.train(steps=5) == example.train(steps=5)        # nothing depends on the order of threads

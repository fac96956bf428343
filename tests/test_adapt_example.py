"""The operators around the frozen convolutions run together, as examples/adapt_stage.py uses them."""
import importlib.util
import os

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.gpu
def test_the_example_learns_its_teacher():
    spec = importlib.util.spec_from_file_location("adapt_stage", os.path.join(ROOT, "examples", "adapt_stage.py"))
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    losses = example.main(40)
    assert all(loss == loss for loss in losses) and losses[-1] < 0.5 * losses[0], losses

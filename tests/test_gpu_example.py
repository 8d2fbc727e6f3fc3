"""The example that trains with both losses on a mesh: they fall."""
import importlib.util
import os

import pytest

pytestmark = pytest.mark.gpu

PATH = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "distill_step.py")


def test_the_losses_fall():
    spec = importlib.util.spec_from_file_location("distill_step", PATH)
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    history = example.main(12)
    first, last = history[0], history[-1]
    assert last[0] < first[0] - 0.05 and last[1] < first[1] - 0.05, (first, last)

"""The example runs its parts together and learns: the loss of its synthetic histories begins at a coin's (0.69) and falls."""
import importlib.util
import os

import pytest

pytestmark = pytest.mark.gpu


def test_history_model_learns():
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "history_model.py")
    spec = importlib.util.spec_from_file_location("history_model", path)
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    losses = module.main(["--steps", "120", "--items", "2000"])
    assert all(x == x for x in losses)
    assert sum(losses[:5]) / 5 > 0.6
    assert sum(losses[-20:]) / 20 < 0.5

"""The operators that learn vectors and the index that answers from them, together."""
import importlib.util
import os

import pytest

pytestmark = pytest.mark.gpu


def test_learnt_projection_is_searched():
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "learn_projection.py")
    spec = importlib.util.spec_from_file_location("learn_projection", path)
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    losses, before, after = module.main(["--vectors", "20000", "--steps", "60"])
    assert losses[-1] < losses[0] - 2 and after > before + 0.2

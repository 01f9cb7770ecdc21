"""The operators together, as examples/gated_mlp.py uses them: training through frozen NVFP4 weights, serving with
4-bit weights."""
import importlib.util
import os

import pytest

pytestmark = pytest.mark.gpu


def test_example():
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "gated_mlp.py")
    spec = importlib.util.spec_from_file_location("gated_mlp", path)
    mod = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(mod)
    losses, errors = mod.main(["--hidden", "256", "--inner", "704", "--tokens", "300", "--steps", "8"])
    # Adam moves every weight by about its rate a step, against the gradient's sign: the loss falls
    assert losses[-1] < losses[0]
    # E2M1 has two significant bits: a value is off by a fifth of itself at most, but for the smallest of a block and
    # what saturates; the products add up three such errors
    assert errors["gate"] < 0.2 and errors["down"] < 0.2
    assert errors["prompt"] < 0.5 and errors["tokens"] < 0.5

"""The example that prunes a layer and distils it back, end to end."""
import importlib.util
import os

import pytest

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_recovery_example_recovers():
    spec = importlib.util.spec_from_file_location("recover_pruned_layer", os.path.join(ROOT, "examples", "recover_pruned_layer.py"))
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    result = example.recover(steps=20)
    assert bin(result["kept"]).count("1") == 4
    losses = result["losses"]
    assert losses[-1] < 0.5 * losses[0]                      # gradient descent on the loss it differentiates
    assert result["after"][0] > result["before"][0] and result["after"][1] > result["before"][1]

"""The example runs end to end: norm, gated block, head, log probabilities and their gradients train a pruned
sub-layer, and its packed form answers as the trained one does."""
import importlib.util
import os

import pytest

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_pruned_feed_forward():
    spec = importlib.util.spec_from_file_location("pruned_feed_forward", os.path.join(ROOT, "examples", "pruned_feed_forward.py"))
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    r = example.main(steps=150)
    assert r["status"] == 0
    # from above the uniform guess to near the chain's own entropy, pruned to 2 of 8 all the while at the end
    assert r["first"] > 5.5 and r["last"] < 2.0
    assert r["floor"] - 0.1 < r["packed"] < r["last"] + 0.2
    assert r["hits"] > 0.75

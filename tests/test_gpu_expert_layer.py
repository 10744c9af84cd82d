"""The example of an expert layer, forward and backward, against float32.

A value rounded to e4m3 is off by at most 2^-4 of itself, 2^-4 / sqrt(3) = 3.6 % in the mean square; independent
roundings of k operands add up to sqrt(k) times that.  The output goes through 4 rounded operands (x, W1, h, W2),
the furthest gradient through 7 (dy, W2, x and W1 through the activation's slope, dup, W1, and bf16 in between): 9.5 %.
"""
import importlib.util
import os

import pytest

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.parametrize("sizes", [dict(tokens=300, topk=2, experts=5, width=256, hidden=384), dict(tokens=64, topk=4, experts=16, width=128, hidden=256)])
def test_expert_layer_and_its_gradients(sizes):
    spec = importlib.util.spec_from_file_location("expert_layer", os.path.join(ROOT, "examples", "expert_layer.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    off, _, _ = m.run(**sizes)
    assert off["y"] < 0.036 * 2 and off["y of one token"] < 0.036 * 2 * 1.5      # one token: few samples of the mean
    assert max(off.values()) < 0.095 * 1.5 and len(off) == 6
    assert all(v > 0.01 for k, v in off.items())                                # it did go through e4m3

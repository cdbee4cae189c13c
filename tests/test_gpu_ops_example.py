"""The example that chains the model operators and has the gate judge their outputs."""
import os
import sys

import pytest
import torch

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.parametrize("tokens,width,out", [(300, 512, 640), (7, 1000, 385)])
def test_example_passes_the_sound_ways_and_fails_the_mistakes(tokens, width, out):
    sys.path.insert(0, os.path.join(ROOT, "examples"))
    try:
        import eight_bit_layer
    finally:
        sys.path.pop(0)
    status, passed, grads, order = eight_bit_layer.main(tokens, width, out, repeats=4, log=lambda *_: None)
    assert status == 0
    for name, ok in passed.items():
        assert ok == (not name.startswith("mistake")), name
    assert sorted(order) == sorted(n for n, ok in passed.items() if ok)
    assert grads["x"].shape == (tokens, width) and grads["W"].shape == (out, width)
    assert all(bool(torch.isfinite(g.float()).all()) for g in grads.values())

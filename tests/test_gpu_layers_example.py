"""The example that runs the layer calls and the collective's local work together: its loss falls, and runs are alike bit by bit."""
import os
import sys

import pytest

pytestmark = pytest.mark.gpu

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


def test_two_layers_learn():
    import train_layers
    losses = train_layers.train(steps=40, ranks=2, rows=96, sizes=(70, 160, 33), verbose=False)
    assert all(l == l for l in losses)
    assert sum(losses[-5:]) < 0.4 * sum(losses[:5])
    assert train_layers.train(steps=3, ranks=2, rows=96, sizes=(70, 160, 33), verbose=False) == losses[:3]

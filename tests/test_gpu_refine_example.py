"""The example that trains and serves a refiner of rendered views runs, learns,
and serves what it trained."""
import os
import sys

import pytest

pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))),
                                "examples"))


def test_refiner_example_learns_and_serves():
    import refine_views
    losses, apart = refine_views.main(steps=40, width=64, height=48,
                                      say=lambda *a: print(*a, flush=True))
    # the frames differ by far more than the network's 16-bit rounding
    assert losses[0] > 1e-4
    assert losses[-1] < 0.5 * losses[0]
    # serving runs the same kernels on the same values
    assert apart < 1e-6

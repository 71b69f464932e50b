"""The example that uses the 4-bit operators and the routing together: it learns, and it serves what it learnt."""
import importlib.util
import os

import pytest

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.parametrize("fmt", ["e4m3_16", "e8m0_32"])
def test_the_example_learns_and_serves(fmt):
    spec = importlib.util.spec_from_file_location("fp4_experts_example", os.path.join(ROOT, "examples", "fp4_experts.py"))
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    losses, apart, size = example.run(steps=60, format=fmt)
    assert sum(losses[-5:]) / 5 < 0.8 * sum(losses[:5]) / 5
    if fmt == "e8m0_32":            # no scale spans tokens: a token's result does not depend on the others'
        assert apart == 0.0
    assert size > 0.0

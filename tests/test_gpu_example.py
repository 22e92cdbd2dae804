"""The example that runs the operators together: both of its ways of training learn the chain."""
import importlib.util
import math
import os

import pytest

pytestmark = pytest.mark.gpu
PATH = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "tied_embedding.py")


@pytest.mark.parametrize("optimizer", ["adamw", "qadam"])
def test_the_example_learns(optimizer):
    spec = importlib.util.spec_from_file_location("tied_embedding", PATH)
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    losses = example.main(["--optimizer", optimizer, "--steps", "300"])
    assert len(losses) == 300 and all(math.isfinite(x) for x in losses)
    # from what a model that knows nothing has (log 1000) at least half the way to the chain's own entropy (log 4)
    assert losses[0] > math.log(1000) and sum(losses[-10:]) / 10 < 0.5 * (math.log(1000) + math.log(4))

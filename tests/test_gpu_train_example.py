"""The example training run: lookup, gradient, reducer and orthogonalised update together.  The chain's entropy is
log 4 = 1.39 and a model that knows nothing is at log 1000 = 6.9 or above."""
import importlib.util
import os

import pytest

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.parametrize("format", ["binary", "ternary"])
def test_loss_falls(format):
    spec = importlib.util.spec_from_file_location("train_small", os.path.join(ROOT, "examples", "train_small.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    losses = m.main(["--steps", "60", "--format", format])
    assert all(x == x for x in losses)
    assert sum(losses[-5:]) / 5 < sum(losses[:5]) / 5 - 1.0

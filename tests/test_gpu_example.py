"""The example of a whole training step runs, learns, and sends only part of
the gradient."""
import math

import pytest

pytestmark = pytest.mark.gpu

pytest.importorskip("torch")
from examples import bigram_step  # noqa: E402


def test_bigram_model_learns():
    losses, density = bigram_step.train(40, 2, tokens=512)
    assert losses[0] > math.log(bigram_step.VOCAB) - 0.5
    assert losses[-1] < losses[0] - 1.0
    assert 0.0 < density < 1.0
    assert all(math.isfinite(v) for v in losses)

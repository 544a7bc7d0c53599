"""examples/decoder_step.py reports a layer that goes wrong."""
import math

import pytest

from tests.test_gpu_decoder import _example

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("value", [math.nan, math.inf, 100.0])
@pytest.mark.parametrize("node", [0, 5, -1])
def test_results_that_are_no_numbers_are_reported(monkeypatch, value, node):
    ex = _example()
    step = ex.DecoderAttention.step

    def spoilt(self, *args):
        y = step(self, *args)
        y[node, 3] = value
        return y

    monkeypatch.setattr(ex.DecoderAttention, "step", spoilt)
    assert not ex.main(["--hidden", "256", "--heads", "4", "--kv-heads", "2", "--head-dim", "32"]) <= 0.02

"""Convolutions, normalisation, ReLU and Muon together: the example learns its ten patterns in every storage type and layout."""
import math

import pytest

from paper_2106_06998_amd import train_example

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,channels_last", [("f32", False), ("bf16", True), ("f16", False)])
def test_the_example_learns(dtype, channels_last):
    print("[gpu-case] train_example", dtype, "channels-last" if channels_last else "planes", flush=True)
    losses, wrong = train_example.train(40, dtype, channels_last, report=lambda *a: None)
    # chance is a loss of log 10 and an error rate of 0.9
    assert all(math.isfinite(v) for v in losses)
    assert sum(losses[-5:]) / 5 < 0.5 * math.log(10) and wrong < 0.3

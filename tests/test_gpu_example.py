"""The decoder of examples/decoder.py, trained and served."""
import importlib.util
import os

import pytest

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_decoder_trains_and_serves():
    spec = importlib.util.spec_from_file_location(
        "decoder", os.path.join(ROOT, "examples", "decoder.py"))
    decoder = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(decoder)
    losses, worst, right = decoder.main(["--steps", "40", "--requests", "9", "--new", "10"])
    # From ln 256 = 5.55 towards the table's entropy, 0.1 * 5.55 + 0.33 nats.
    assert losses[0] > 5.0 and losses[-1] < 0.5 * losses[0]
    # Both ways round their weights and outputs to 8 bits of bfloat16, from
    # values that differ in their own last bit: logits of a few units.
    assert worst < 0.25
    assert right > 0.8

"""The example that trains a small model on packed blocks: it learns, and packing changes nothing for a sequence."""
import importlib.util
import os

import pytest

pytestmark = pytest.mark.gpu


def test_the_example_learns_and_packed_sequences_do_not_notice_each_other():
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "packed_layers.py")
    spec = importlib.util.spec_from_file_location("packed_layers", path)
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    losses, apart = example.main(steps=40, quiet=True)
    assert losses[-1] < 0.5 * losses[0]
    # 16-bit activations in two layers, added to a residual stream in 32 bits: a few roundings of 2^-8 of a layer's output
    assert apart < 4 * 2.0 ** -8

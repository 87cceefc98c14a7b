"""The example model, whose layers are made of the library's operators: it learns, and decoding from kept states gives the logits of
the whole sequence at once.  Tolerance: between the two ways activations are rounded to bfloat16 at the same places, so that
they differ where sums of floats in another order round to a neighbour (2^-8), passed on through two layers of residual sums: a few
hundredths of the logits' spread; 0.1 is allowed."""
import importlib.util
import os

import pytest

pytestmark = pytest.mark.gpu


def test_the_example_learns_and_decodes():
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "decay_language_model.py")
    spec = importlib.util.spec_from_file_location("decay_language_model", path)
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    first, last, entropy, off = m.main(["--steps", "60"])
    assert first > 5.0  # near log 256 at first
    assert entropy < last < (first + entropy) / 2
    assert off < 0.1

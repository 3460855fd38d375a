"""The example runs the sequence operators and AdamW together: it learns, and its streaming form agrees."""
import os
import sys

import pytest

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("bits", (32, 8))
def test_selective_raster_learns_and_streams(bits):
    import selective_raster
    r = selective_raster.train("tiny_ff", width=48, states=8, steps=60, lr=1e-2, state_bits=bits, say=lambda s: None)
    assert r["last"] < 0.8 * r["first"], r
    # the sum over steps of values rounded to bfloat16 (2^-8 of each, at random), through two products of bfloat16
    assert r["apart"] < 2 ** -6, r

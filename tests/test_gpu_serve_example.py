"""The example of a served attention layer runs, from compressed weights through a captured step, and
stays near the unquantised layer.

What it may be off by, with every rounding at its largest and independent: activations and keys in
E4M3 are off by up to 2^-4 of a value, 2^-4 / sqrt(3) root mean square over a half unit, and less
where a value lies high in its binade; two quantised projections, the scores (a relative change of
a weight by what the score moves) and the values add up in squares to under 4 such errors, below
8 %.  A step that mixed up a page, a slot or a scale is off by the size of the result.
"""
import os
import sys

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.mark.parametrize("cache", ["e4m3", "int8"])
def test_served_layer_stays_near_the_plain_one(cache):
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    sys.path.insert(0, os.path.join(root, "examples"))
    try:
        import serve_attention_layer as example
    finally:
        sys.path.pop(0)
    assert example.main(["--steps", "70", "--cache", cache]) < 0.08

"""The example of a whole served layer runs, from compressed weights through a captured step, and
what the layer adds to the residual stream stays near what the unquantised layer adds.

What it may be off by, with every rounding at its largest and independent: the attention's share as
in its own example, below 8 % of it.  The MLP's operands in INT8 rows are off by half a code, 1 / 254 of
a row's largest value; rows of some thousand near-normal values have that at 4 or 5 of their root mean
square (the activation's products at 10 or so), so a value is off by 2 % (4 %) of that at most, 1.2 % (2.3 %)
root mean square; a product keeps that ratio, and the gated product of two such halves adds theirs: below
6 % in squares with the attention's error that comes in by the residual stream.  BF16 sums of the stream
add 2^-8 of the stream, several times what the layer adds at worst: 2 %.  In all below 12 %.  A step that
mixed up a position, a scale or a half is off by the size of the result.
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
        import serve_transformer_layer as example
    finally:
        sys.path.pop(0)
    assert example.main(["--steps", "70", "--cache", cache]) < 0.12

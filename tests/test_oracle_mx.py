"""Pins of the MXFP4 oracle: hand cases of the rounding, exactness of the values, and the layouts' bijection."""
import math

import numpy as np
import pytest

from oracle import mx


@pytest.mark.parametrize("v,code", [(0.0, 0), (-0.0, 8), (0.25, 0), (0.2500001, 1), (0.5, 1), (0.75, 2), (0.7499, 1), (1.25, 2), (1.75, 4),
                                    (2.5, 4), (2.51, 5), (3.5, 6), (5.0, 6), (5.01, 7), (6.0, 7), (7.99, 7), (-5.01, 15)])
def test_rounding(v, code):
    assert mx.round_value(v) == code


@pytest.mark.parametrize("block,scale", [([1.0], 125), ([4.0], 127), ([7.9], 127), ([8.0], 128), ([0.0, -0.0], 0), ([2.0 ** -126], 0),
                                         ([2.0 ** -140], 0), ([2.0 ** -124], 1), ([3.0e38], 252), ([math.inf, 1.0], 255), ([math.nan], 255)])
def test_power_of_two(block, scale):
    assert mx.round_block(block)[1] == scale


def test_values_of_the_format_come_back():
    """Every code under every scale that rounding can give: a block that holds a 4 or a 6 rounds to itself."""
    codes = np.array([[c for c in range(16)] * 2], np.uint8)
    for s in range(0, 253):
        scales = np.array([[s]], np.uint8)
        again = mx.quantize(mx.values(codes, scales))
        assert np.array_equal(again[0], codes) and np.array_equal(again[1], scales)


@pytest.mark.parametrize("rows,cols", [(1, 32), (31, 96), (32, 64), (33, 256), (64, 288), (70, 512)])
def test_tile_layout_is_a_bijection(rows, cols):
    """Every byte of the matrix is somewhere, once; the rest is filling."""
    rng = np.random.default_rng(rows * 1000 + cols)
    codes = rng.integers(1, 8, (rows, cols), np.uint8)                # no zero codes: filling is told apart
    scales = rng.integers(1, 100, (rows, cols // 32), np.uint8)
    c, s = mx.pack_tiles(codes, scales)
    packed, filled = mx.pack_rows(codes, scales)
    assert sorted(c[c != 0].tolist()) == sorted(packed.reshape(-1).tolist())
    assert sorted(s[s != 127].tolist()) == sorted(scales.reshape(-1).tolist())
    assert (filled[:, cols // 32:] == 127).all()

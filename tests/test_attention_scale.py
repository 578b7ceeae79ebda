"""Scales that attention takes (no GPU is touched: every call ends before a launch): what the kernels make of them, to base 2 and in the cache's units of 2^69, has to be
finite, as have its power of two above and its reciprocal in normal numbers."""
import math

import numpy as np
import pytest

torch = pytest.importorskip("torch")

import paper_2504_08009_amd as oz
from test_attention_arguments import P, attention, cache, ref, rows, sequences


def step(scale):
    return oz.lib().oz2_kv4_attention(ref(cache()), ref(sequences(tokens=0)), 8, scale, ref(rows(P, 512, 64)), ref(rows(P << 1, 512, 64)), None)


@pytest.mark.parametrize("call,most,code", [(lambda s: attention(scale=s), 2.0 ** 126, -7), (step, 2.0 ** 55, -4)], ids=["prompts", "cache"])
def test_scales_up_to_a_power_of_two(call, most, code):
    up = float(np.nextafter(np.float32(most), np.float32(math.inf)))
    for scale in (2.0 ** -149, 1e-30, 0.125, 1.0, 1e10, most / 2, most):
        assert call(scale) == 0
    for scale in (up, 2 * most, 3.4e38, math.inf, math.nan, 0.0, -0.0, -1.0, -most):
        assert call(scale) == code


def test_what_becomes_of_the_largest():
    for most, units in ((2.0 ** 126, 1.0), (2.0 ** 55, 2.0 ** 69)):
        scale2 = np.float32(np.float32(most * math.log2(math.e)) * np.float32(units))
        above = 2.0 ** math.ceil(math.log2(scale2))
        assert np.isfinite(scale2) and above <= 2.0 ** 127 and (units == 1.0 or 1 / scale2 >= 2.0 ** -126)

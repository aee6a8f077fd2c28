"""Pins of the oracle of the 8-bit cache at the top of its range: whatever finite value comes in, what its code stands for is a
finite bf16 number."""
import numpy as np
import pytest

from oracle import kvra_oracle as orc
from oracle import lowbit

TOP = 2.0 ** 120
LARGEST = (2.0 - 2.0 ** -7) * 2.0 ** 127        # of bf16


@pytest.mark.parametrize("value,code", [
    (240.0, 0x77), (241.0, 0x77), (247.0, 0x77), (248.0, 0x77), (250.0, 0x77), (255.0, 0x77), (256.0, 0x77), (1e6, 0x77),
    (225.0, 0x76), (224.0, 0x76), (1.0, 0x38), (np.nan, 0x7F), (np.inf, 0x7F),
])
def test_codes_with_the_largest_scale(value, code):
    assert list(lowbit.e4m3_codes(np.array([value, -value]) * TOP, 120))[0] == code
    if np.isfinite(value):
        assert list(lowbit.e4m3_codes(np.array([-value]) * TOP, 120))[0] == code | 128


def test_the_scale_below_it_still_has_every_code():
    assert list(lowbit.e4m3_codes(np.array([448.0, 256.0, 447.0]) * TOP / 2, 119)) == [0x7E, 0x78, 0x7E]


@pytest.mark.parametrize("gain", [1.0, 2.0 ** 0.5])       # (a rotated K: up to sqrt(2) times what came in)
def test_a_cache_of_the_largest_values_is_finite_in_bf16(gain):
    new = np.full((5, 2, 64), LARGEST * gain)
    new[:, 1] = -LARGEST * gain
    new[2, 0, :4] = [248 * TOP, 240 * TOP, 7.0 * TOP, 0.0]
    cache, scale = np.zeros((64, 2, 64), np.uint8), np.zeros((1, 2), np.uint8)
    lowbit.append_rows(cache, scale, np.full((3, 2, 64), 1.75 * 2.0 ** 126), 0)      # (held rows: rescaled from 118)
    lowbit.append_rows(cache, scale, new, 3)
    assert np.all(scale == 247)
    values = lowbit.cache_values(cache, scale)[:8]
    assert np.all(values[:3] == 1.75 * 2.0 ** 126)
    assert np.abs(values).max() == 240 * TOP and list(values[5, 0, :4] / TOP) == [240.0, 240.0, 7.0, 0.0]
    assert np.array_equal(orc.bf16_bits_to_f64(orc.f64_to_bf16_bits(values)), values)

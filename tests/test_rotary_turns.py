"""Frequencies as fractions of a turn (scoot_rotary_turns): against exact arithmetic (no GPU)."""
from fractions import Fraction

import numpy as np
import pytest

from test_serving_binding import S, lib  # noqa: F401

# pi to 99 decimals
PI = Fraction(3141592653589793238462643383279502884197169399375105820974944592307816406286208998628034825342117067, 10 ** 99)


def _off(got, frequency, position=1):
    """How far position * got is from the angle, in units of 2^-64 of a turn."""
    off = (position * int(got) - position * Fraction(float(frequency)) / (2 * PI) * (1 << 64)) % (1 << 64)
    return min(off, (1 << 64) - off)


@pytest.mark.parametrize("frequencies", [
    [1.0, 0.5, 2.0 ** -20, 1e-4, -1e-9, 1e-25, 5e-324, 0.0, -0.0],
    [2 * np.pi * 0.25, 2 * np.pi * 3.5, -2 * np.pi * 0.125, np.pi, 2 * np.pi, np.nextafter(2 * np.pi, 0)],
    [1000.0, 12345.678, -1e6, 2.0 ** 30, -(2.0 ** 30) + 0.125, 2.0 ** 40 / 3],
    list(10000.0 ** (-np.arange(64) / 64)), list(500000.0 ** (-np.arange(32) / 32))])
def test_turns_are_off_by_a_unit_at_most(S, frequencies):
    """One rounding to whole units, and what two words of 1 / 2 pi leave out (2^-106 of the turns, 2^-67 of one here)."""
    for f, got in zip(frequencies, S.scoot_rotary_turns(np.array(frequencies)).tolist()):
        assert _off(got, f) <= 1, f


def test_angles_at_the_farthest_positions(S):
    """As the header says: within 2^-33 of a turn of position times frequency."""
    f = np.concatenate([S.scoot_rotary_frequencies(128), S.scoot_rotary_frequencies(64, 500000.0, "parts", 8.0, original_len=8192), [1000.0, -77.7]])
    for x, got in zip(f, S.scoot_rotary_turns(f).tolist()):
        for p in (2 ** 31 - 1, -2 ** 31, 1 << 20):
            assert _off(got, x, p) <= 1 << 31


def test_frequencies_of_any_size_have_a_fraction(S):
    f = np.array([1e300, -1e308, 2.0 ** 60, 1.7976931348623157e308])
    assert S.scoot_rotary_turns(f).dtype == np.uint64   # (their fractions are as good as the doubles: no digits are left)

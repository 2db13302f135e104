"""How exact the rotation's steps are: what include/netkv.h says of an angle rests on it.  No GPU here."""
import math
from fractions import Fraction

import pytest

from tests.test_chunk_host import lib  # noqa: F401

PI = Fraction(314159265358979323846264338327950288419716939937510, 10 ** 50)


@pytest.mark.parametrize("frequencies", [
    [500000.0 ** (-p / 64) for p in range(64)], [1.0 - p / 100 for p in range(64)],
    [6.2 - p / 1000 for p in range(64)], [4.0 + p / 50 for p in range(64)], [1e-9 * (p + 1) for p in range(64)]])
def test_a_step_is_the_part_of_a_turn(lib, frequencies):  # noqa: F811
    """To 2^-52 of itself and one unit: position t is then off by t * frequency * 2^-52 of a radian, and
    by less than 2^-30 of one for the unit, at the last of 2^31 positions."""
    r = lib.Rotary(64, frequencies=frequencies)
    for f, step in zip(frequencies, r.step):
        want = Fraction(f) / (2 * PI) * 2 ** 64
        assert abs(step - want) <= want * Fraction(1, 2 ** 52) + 1
        assert 2 ** 31 * 2 * math.pi / 2 ** 64 < 2.0 ** -30

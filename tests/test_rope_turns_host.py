"""The rounding of tg_rope_turns (CPU only)."""
import math
from fractions import Fraction

import pytest

from paper_2606_06302_amd import tangram as tg
from test_rope_host import TWO_PI, fraction_of


def off_by(theta, turns):
    want = Fraction(theta) / TWO_PI
    off = abs(fraction_of(turns) - (want - math.floor(want)))
    return min(off, 1 - off)


UNIT = 2 * math.pi / 2 ** 64
THETAS = [s * UNIT * k for s in (1, -1) for k in (1, 2, 3, 5, 1001, 12345677, 2 ** 40 + 1)] + [
    -5e-324, -1e-30, math.pi, -math.pi, math.pi * (1 + 2 ** -40), 4.0, 5.0, 6.2, -1.0, -0.7]


@pytest.mark.parametrize("theta", THETAS)
def test_the_nearest_fraction(theta):
    """Half a step of the fraction (2^-65), a quarter more from the whole turns' subtraction, and what the quotient by 2 pi
    loses of theta's own size (three roundings of 2^-64: 2 pi, the quotient, and one to spare)."""
    turns = tg.tg_rope_turns([theta])[0]
    assert off_by(theta, turns) <= Fraction(3, 4) / 2 ** 64 + 3 * abs(Fraction(theta)) / TWO_PI / 2 ** 64


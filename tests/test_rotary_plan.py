"""The turns that a rotation's plan holds (eas_rotary_make, host only): against the quotient of the frequency by 2 pi in whole
numbers, of every size that is taken."""
from fractions import Fraction

import numpy as np
import pytest

from paper_2609_31551_amd import eas
from test_attention_abi import UNSUPPORTED
from test_paged_abi import PI, make

TURN = Fraction(2 * PI, 10 ** 59)                     # pi's own rest is below 10^-59: 2^-136 of the largest quotient


def off(step, f):
    """Distance of a step from f / (2 pi), in 2^-64 of a turn, whole turns aside."""
    d = (step - Fraction(f) / TURN * 2 ** 64) % 2 ** 64
    return min(d, 2 ** 64 - d)


@pytest.mark.parametrize("size", [-1070, -300, -140, -129, -128, -127, -70, -66, -65, -64, -63, -30, -1, 0, 1, 5, 10, 20, 31, 40,
                                  50, 52, 53, 54, 56, 57, 58, 59])
def test_steps_of_every_size(size):
    """Rounding, and 1 / (2 pi) to 128 bits: half a step and 2^-68 of a turn."""
    rng = np.random.default_rng(size + 2000)
    freqs = [float(np.ldexp(x, size)) for x in [1.0, 1.5, 2.0 - 2.0 ** -52] + list(rng.uniform(1, 2, 29))]
    freqs += [-f for f in freqs]
    status, r = make(freqs)
    assert status == eas.EAS_OK
    for f, step in zip(freqs, r.step):
        assert off(step, f) <= Fraction(1, 2) + Fraction(1, 16), f


def test_quarter_turns_and_whole_ones():
    freqs = [float(np.pi * k / 2) for k in range(-4, 4)] + [0.0, -0.0, 5e-324, 2 * np.pi * 12345, -2 * np.pi, 1e18, -1e18, 1e-40]
    status, r = make(freqs)
    assert status == eas.EAS_OK
    for f, step in zip(freqs, r.step):
        assert off(step, f) <= Fraction(9, 16), f
    assert r.step[8] == r.step[9] == r.step[10] == 0


@pytest.mark.parametrize("f", [2.0 ** 60, -2.0 ** 60, 1e300, -1.7e308])
def test_frequencies_that_are_not_taken(f):
    assert make((1.0,) * 7 + (f,))[0] == UNSUPPORTED
    assert make((1.0,) * 7 + (float(np.nextafter(np.copysign(2.0 ** 60, f), 0)),))[0] == eas.EAS_OK

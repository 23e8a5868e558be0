"""The table of frequencies for fast pairs, in units of 2^-64 of a turn, against 60 digits."""
import decimal
import fractions

import pytest

from paper_2608_13524_amd import dartree as D
from tests.test_more_abi import PI

d = decimal.Decimal


def off(turn, radians):
    """How far a table's entry is from the fraction of a turn in `radians`, in units of 2^-64, either way round."""
    with decimal.localcontext(decimal.Context(prec=60)):
        x = fractions.Fraction(radians / (2 * PI))
    x = (turn - x * (1 << 64)) % (1 << 64)
    return min(x, (1 << 64) - x)


@pytest.mark.parametrize("radians", [0.0, 1.0, -1.0, 2.0, 3.5, 100.0, -100.0, 12345.678, 1e6, -1e6, 2.0 ** 31 + 0.25, 3e9, 1e12, -7e15,
                                     6.283185307179586, 5e-324, 1e-10])
def test_any_frequency_within_a_unit(radians):
    """The quotient by 2 pi in twice 64 bits: what is left of it is rounded to a unit, and once before, half a unit each."""
    got = D.rotary_turns_of([radians], "cpu").tolist()[0]
    assert off(got, d(radians)) <= 1


def test_frequencies_past_all_precision_are_some_number():
    for radians in (1e30, -1e300, 1.7e308):
        assert len(D.rotary_turns_of([radians], "cpu")) == 1


@pytest.mark.parametrize("rot,base", [(2, 10000.0), (80, 500000.0), (128, 10000.0), (512, 1e6), (64, 1e-6), (128, 0.5)])
@pytest.mark.parametrize("rule,factor,low,high,length", [(0, 1.0, 0.0, 0.0, 0), (1, 8.0, 0.0, 0.0, 0), (1, 1e-3, 0.0, 0.0, 0),
                                                         (2, 4.0, 0.0, 0.0, 0), (3, 4.0, 1.0, 32.0, 4096), (3, 8.0, 1.0, 4.0, 8192)])
def test_rules_within_two_units(rot, base, rule, factor, low, high, length):
    """Two units of f radians where f > 1, else two: a frequency is made in 64 bits of mantissa, in which the power, its
    rounded exponent (at most 14 / 2 of a unit of f here) and two or three products are off by less than 10 units of f,
    a sixth of which are turns; one more unit as above."""
    got = D.rotary_turns(rot, base, D.RotaryScaling(rule, factor, low, high, length), device="cpu")
    with decimal.localcontext(decimal.Context(prec=60)):
        b = d(base)
        if rule == 2 and rot > 2:
            b *= d(factor) ** (d(rot) / d(rot - 2))
        for i, t in enumerate(got.tolist()):
            f = b ** (d(-2 * i) / d(rot))
            if rule == 1:
                f /= d(factor)
            if rule == 3:
                s = min(max((length * f / (2 * PI) - d(low)) / (d(high) - d(low)), d(0)), d(1))
                f *= s + (1 - s) / d(factor)
            assert off(t, f) <= 2 * max(f, d(1)), i

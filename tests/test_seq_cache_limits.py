"""The paged cache's host arithmetic at its limits (CPU only)."""
import ctypes as C
from decimal import Decimal, getcontext
from fractions import Fraction

import pytest

from paper_2509_20883_amd import recis as R


def _pi(bits):
    """pi 2^bits, by Machin's formula in whole numbers."""
    one = 1 << (bits + 16)

    def atan_inv(n):
        total, term, k, sign = 0, one // n, 1, 1
        while term:
            total += sign * (term // k)
            term //= n * n
            k, sign = k + 2, -sign
        return total

    return (4 * (4 * atan_inv(5) - atan_inv(239))) >> 16


BITS = 600
TWO_PI = Fraction(2 * _pi(BITS), 1 << BITS)


def _off(got, f):
    """How far a fraction of 2^64 is from the frequency's, in units of 2^-64 turns, around the turn."""
    want = f / TWO_PI
    d = Fraction(got, 1 << 64) - (want - want.__floor__())
    return abs(d - round(d)) * 2 ** 64


FREQS = [0.0, 1.0, -1.0, 6.25, 6.283185307179586, 100.0, -100.0, 1e5, -1e5, 12345.678, 1e9, 1e15, 2.0 ** 63, 1.7e30, -1.2345 * 2.0 ** 100,
         2.0 ** 127 * 1.999, 0.1, 1e-3, 2.0 ** -60, 1.7 * 2.0 ** -62, 2.0 ** -70, 5e-324]


def test_own_frequencies_are_exact():
    """A frequency is the double that it is, whatever its size: its fraction of a turn is off by the last rounding."""
    got = (C.c_uint64 * len(FREQS))()
    assert R.lib().rs_rotation_turns((C.c_double * len(FREQS))(*FREQS), 0.0, 2 * len(FREQS), got) == R.OK
    for f, g in zip(FREQS, got):
        assert _off(g, Fraction(f)) <= 0.5 + 2.0 ** -20, f


@pytest.mark.parametrize("f", [2.0 ** 128, -2.0 ** 128, 1e300, float("inf"), float("nan")])
def test_frequencies_that_are_refused(f):
    got = (C.c_uint64 * 2)()
    assert R.lib().rs_rotation_turns((C.c_double * 2)(1.0, f), 0.0, 4, got) == R.EINVAL


def test_a_base_whose_powers_are_refused():
    got = (C.c_uint64 * 64)()
    assert R.lib().rs_rotation_turns(None, 5e-324, 128, got) == R.EINVAL  # up to 2^1057


@pytest.mark.parametrize("base,rotary", [(10000.0, 128), (500000.0, 64), (1.0, 6), (1e300, 32), (0.5, 48)])
def test_frequencies_of_a_base(base, rotary):
    """base^(-2 i / rotary) in 64 bits: the power is off by less than its last, 2^-63 of itself, its exponent by 2^-64 of itself, which
    is ln f of the power; then the last rounding.  One unit is never passed from base 1 on."""
    getcontext().prec = 60
    got = (C.c_uint64 * (rotary // 2))()
    assert R.lib().rs_rotation_turns(None, base, rotary, got) == R.OK
    for i in range(rotary // 2):
        f = (Decimal(base).ln() * Decimal(-2 * i) / Decimal(rotary)).exp()
        bound = 0.5 + float(f) / 6.28 * (2 + abs(float(f.ln())))
        assert _off(got[i], Fraction(f)) <= bound and (base < 1 or bound < 1), i

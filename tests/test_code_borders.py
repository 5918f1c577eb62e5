"""8-bit codes by one remainder step (Quotient in csrc/pp_paged.cu) are those of the rounded quotient, in exact arithmetic.

With y = 1 / scale, q = x y and q' = q + (x - q scale) y, each rounded to a float, q' is within 2^-22 of a unit of its last place of
x / scale before its own rounding.  So it can round to another float than x / scale does only where the quotient is that near the middle
of two floats, and that matters only next to a border of two codes.  Next to a border C 2^g (C odd, 2^n <= C < 2^(n+1)) a middle is
C 2^g (1 +- half a unit); in units of the border's last bit times the scale's, x - C S is whole and half a unit is S 2^(n-24) for a scale of
significand S: they meet within 2^-22 of a unit, 2^(n-22), only for S within 4 of a multiple of 2^(24-n).  All of these are tried."""
from fractions import Fraction as Fr

import pytest


def _rounded(n, d):
    """n / d > 0 to 24 bits, ties to even: a fraction."""
    e = n.bit_length() - d.bit_length()
    if (n << max(-e, 0)) < (d << max(e, 0)):
        e -= 1
    shift = 23 - e
    n, d = n << max(shift, 0), d << max(-shift, 0)
    q, r = divmod(n, d)
    q += 2 * r > d or (2 * r == d and q & 1)
    return Fr(q << max(-shift, 0), 1 << max(shift, 0))


def _round(v):
    return -_rounded(-v.numerator, v.denominator) if v < 0 else _rounded(v.numerator, v.denominator) if v else v


def _borders(kind):
    if kind == "int8":
        return [Fr(2 * i + 1, 2) for i in range(127)]
    codes = [Fr(c & 7, 512) if c < 8 else (1 + Fr(c & 7, 8)) * Fr(2) ** ((c >> 3) - 7) for c in range(127)]
    return [(a + b) / 2 for a, b in zip(codes, codes[1:])]


@pytest.mark.parametrize("kind", ["int8", "e4m3"])
def test_one_step_is_on_the_side_of_the_quotient(kind):
    tried = 0
    for border in _borders(kind):
        odd = border.numerator // (border.numerator & -border.numerator)
        n = odd.bit_length() - 1
        for j in range(max(1, 1 << max(n - 1, 0)), (1 << n) + 1):
            for off in range(-4, 5):
                significand = (j << (24 - n)) + off
                if not 1 << 23 <= significand < 1 << 24:
                    continue
                scale = Fr(significand, 1 << 23)
                y, near = _round(1 / scale), _round(border * scale)
                unit = Fr(1, 1 << 24 - 1 - (near.numerator.bit_length() - near.denominator.bit_length()))
                for k in (-2, -1, 0, 1, 2):
                    x = _round(near + k * unit)
                    q = _round(x * y)
                    got, want = _round(q + _round(x - q * scale) * y), _round(x / scale)
                    assert (got < border, got == border) == (want < border, want == border), (border, scale, x)
                    tried += 1
    assert tried > 1000

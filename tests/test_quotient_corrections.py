"""The encoder's quotient x / scale: a product with the rounded reciprocal and two corrections, against exact arithmetic.

Every step is done in rational arithmetic and rounded to float32 as the instruction does it; the result has to be the correctly
rounded quotient wherever its e4m3 code is not 0 anyway, for any scale from 2^-90 to 2^120.  Among the cases: quotients at and next
to the rounding boundaries of e4m3, scales next to sixteenths (where one correction would not do), zeros of both signs.
"""
from fractions import Fraction

import numpy as np

F = np.float32


def _round(x: Fraction, zero=F(0.0)) -> np.float32:
    """Nearest float32, ties to even, of a rational; `zero` is what an exact 0 gives."""
    if x == 0:
        return zero
    mag = abs(x)
    e = max(-126, mag.numerator.bit_length() - mag.denominator.bit_length())
    while mag >= Fraction(2) ** (e + 1):
        e += 1
    while e > -126 and mag < Fraction(2) ** e:
        e -= 1
    n = mag / Fraction(2) ** (e - 23)
    k = n.numerator // n.denominator
    rest = n - k
    if rest > Fraction(1, 2) or (rest == Fraction(1, 2) and k % 2):
        k += 1
    return F(np.copysign(float(k) * 2.0 ** (e - 23), float(1 if x > 0 else -1)))


def _fma(a, b, c):
    exact = Fraction(float(a)) * Fraction(float(b)) + Fraction(float(c))
    if exact == 0:   # a sum of zeros is -0 where both are, an exact difference +0
        pz = np.signbit(a) ^ np.signbit(b)
        both = pz and np.signbit(c) and float(a) * float(b) == 0 and float(c) == 0
        return F(-0.0) if both else F(0.0)
    return _round(exact)


def _encoder_quotient(x, scale):
    y = _round(1 / Fraction(float(scale)))
    q = _round(Fraction(float(x)) * Fraction(float(y)), F(np.copysign(0.0, x)))
    for _ in range(2):
        q = _fma(F(-_fma(q, scale, F(-x))), y, q)
    return q


def _check(x, scale):
    got, want = _encoder_quotient(x, scale), _round(Fraction(float(x)) / Fraction(float(scale)), F(np.copysign(0.0, x)))
    if abs(float(want)) < 2.0 ** -11:
        assert abs(float(got)) < 2.0 ** -10 and np.signbit(got) == np.signbit(x)
    else:
        assert got == want, (float(x).hex(), float(scale).hex(), float(got).hex(), float(want).hex())


def test_random_quotients():
    rng = np.random.default_rng(0)
    for _ in range(6000):
        scale = F(np.ldexp(rng.uniform(1, 2), int(rng.integers(-90, 100))))
        x = F(float(scale) * rng.uniform(-448, 448) * 2.0 ** -int(rng.integers(0, 18)))
        _check(x, scale)


def test_boundaries_and_scales_next_to_sixteenths():
    rng = np.random.default_rng(1)
    for k in range(16, 32):
        for ulps in (-3, -2, -1, 0, 1, 2, 3):
            scale = F(F(k / 16) * F(2.0) ** int(rng.integers(-60, 60)))
            scale = (scale.view(np.int32) + np.int32(ulps)).view(np.float32)
            for j in range(17, 32, 2):                     # boundaries of e4m3: odd sixteenths
                b = float(j) / 16 * 2.0 ** int(rng.integers(-9, 9))
                x = F(b * float(scale))
                for step in range(-2, 3):
                    v = (x.view(np.int32) + np.int32(step)).view(np.float32)
                    _check(v, scale)
                    _check(F(-v), scale)


def test_zeros_and_bf16_ties():
    rng = np.random.default_rng(2)
    for a in rng.integers(128, 256, 40):                   # amax with a bf16 mantissa: exact ties are common
        scale = F(F(a) / F(448))
        for m in rng.integers(128, 256, 40):
            x = F(np.ldexp(float(m), int(rng.integers(-14, 1))))
            if x <= a:
                _check(x, scale)
        for z in (F(0.0), F(-0.0), F(1e-40), F(-1e-45)):
            _check(z, scale)

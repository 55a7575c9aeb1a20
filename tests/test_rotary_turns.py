"""Frequencies as 64-bit fractions of a turn: the nearest one, whatever the frequency."""
import ctypes
import random
from fractions import Fraction

from paper_2511_13198_amd import pdyattn as P

BITS = 1400


def two_pi():
    """2 pi to 2^-BITS by Machin's formula, 16 atan(1 / 5) - 4 atan(1 / 239) = pi."""
    one = 1 << (BITS + 40)

    def atan_inverse(n):
        power, total, k = one // n, 0, 1
        while power:
            total += power // k if k % 4 == 1 else -(power // k)
            power //= n * n
            k += 2
        return total

    return Fraction(2 * (16 * atan_inverse(5) - 4 * atan_inverse(239)), one)


def test_turns_are_the_nearest_fractions():
    rng = random.Random(1)
    ws = [base ** (-p / n) for base in (1e4, 5e5, 1e6) for n in (32, 64) for p in range(n)]
    ws += [3.7e5, -3.7e5, 1e15, 2.0 ** 52 + 1, 1e-19, 2.0 ** -62, 1e-300, 5e-324, 1e300,
           1.7976931348623157e308, -1.7976931348623157e308, 0.0, -0.0]
    ws += [rng.choice((-1, 1)) * rng.uniform(1, 2) * 2.0 ** rng.randrange(-1022, 1023) for _ in range(300)]
    x, y = (ctypes.c_double * len(ws))(*ws), (ctypes.c_uint64 * len(ws))()
    assert P.lib().attn_rotary_turns(x, len(ws), y) == P.PDY_OK
    turn = two_pi()
    for w, f in zip(ws, y):
        off = abs(Fraction(f, 2 ** 64) - Fraction(w) / turn % 1)
        # half of the last bit, and what 2 pi's own last bits leave
        assert min(off, 1 - off) <= Fraction(1, 2 ** 65) + Fraction(1, 2 ** 120), w

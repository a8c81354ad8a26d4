"""fq_rope_turns against whole numbers: the nearest multiple of 2^-64 of a turn, of every finite frequency."""
from fractions import Fraction

import numpy as np

from paper_2410_09426_amd import binding as fq

BITS = 1400


def _arctan_of_one_over(n):
    """arctan(1 / n) 2^BITS, by its series."""
    term, total, k = (1 << BITS + 32) // n, 0, 0
    while term:
        total += (-term if k & 1 else term) // (2 * k + 1)
        term //= n * n
        k += 1
    return total >> 32


PI = 16 * _arctan_of_one_over(5) - 4 * _arctan_of_one_over(239)              # (Machin) times 2^BITS, to a few units


def nearest(x):
    turns = Fraction(x) * (1 << BITS) / (2 * PI) * 2 ** 64
    return int((turns + Fraction(1, 2)).__floor__()) % 2 ** 64


def test_every_size_of_frequency():
    assert str(PI * 10 ** 40 >> BITS) == "31415926535897932384626433832795028841971"
    r = np.random.Generator(np.random.PCG64(7))
    f = [0.0, -0.0, 1.0, -1.0, 3.0, 6.283185307179586, -6.283185307179586, 100.0, 1e6, 2.0 ** 40, 1e17, 1e308, -1e308, 1.7976931348623157e308, 5e-324, 2.2250738585072014e-308, 1e-12, -1e-30]
    f += [10000.0 ** (-2 * i / 128) for i in range(64)] + [500000.0 ** (-2 * i / 96) for i in range(48)]
    f += np.ldexp(r.uniform(-2, 2, 4000), r.integers(-80, 80, 4000)).tolist() + np.ldexp(r.uniform(-2, 2, 2000), r.integers(-1074, 1023, 2000)).tolist()
    got = fq.fq_rope_turns(np.array(f)).tolist()
    wrong = [(x, g, nearest(x)) for x, g in zip(f, got) if g != nearest(x)]
    assert not wrong, (len(wrong), wrong[:5])

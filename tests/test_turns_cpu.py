"""A frequency as a fraction of a turn (csrc/turns.h) on the CPU, against exact rationals: 2 pi to 98 digits by Machin's formula."""

import ctypes
import math
import os
import random
import subprocess
from decimal import Decimal, getcontext
from fractions import Fraction

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def turn(tmp_path_factory):
    at = tmp_path_factory.mktemp("turns")
    (at / "shim.cpp").write_text('#include "turns.h"\nextern "C" uint64_t turn(double f) { return fsx::turn_per_step(f); }\n')
    subprocess.run(["g++", "-std=c++17", "-O2", "-Wall", "-Werror", "-shared", "-fPIC", "-I",
                    os.path.join(ROOT, "paper_2607_15621_amd", "csrc"), str(at / "shim.cpp"), "-o", str(at / "shim.so")], check=True)
    f = ctypes.CDLL(str(at / "shim.so")).turn
    f.restype, f.argtypes = ctypes.c_uint64, [ctypes.c_double]
    return f


def two_pi():
    getcontext().prec = 100

    def atan(n):
        total, term, i = Decimal(0), Decimal(1) / n, 0
        while abs(term) > Decimal(10) ** -99:
            total += term / (2 * i + 1) * (-1) ** i
            term /= n * n
            i += 1
        return total
    return Fraction(8 * (4 * atan(5) - atan(239)))


TURN = two_pi()


def off(got, freq):
    """How far, in units of 2^-64 of a turn, the nearest way round."""
    d = (got - Fraction(freq) * 2 ** 64 / TURN) % 2 ** 64
    return min(d, 2 ** 64 - d)


@pytest.mark.parametrize("freq", [2.0 ** 20, math.nextafter(2.0 ** 20, 0), 987654.321, 12345.678, 10.0, 1.0, 0.1, 2 * math.pi, math.pi, 1e-4, 2.0 ** -30,
                                  2.0 ** -61, 2.0 ** -62, 20 * 2.0 ** -66, 2.0 ** -66, 2.0 ** -70, 1e-300, 5e-324, 0.0])
def test_known(turn, freq):
    for f in (freq, -freq):
        assert off(turn(f), f) <= Fraction(1, 2) + Fraction(1, 2 ** 44), f
    assert (turn(freq) + turn(-freq)) % 2 ** 64 == 0


def test_every_size(turn):
    rng = random.Random(7)
    for _ in range(20000):
        f = math.ldexp(rng.choice((-1, 1)) * rng.uniform(0.5, 1), rng.randint(-80, 20))
        assert off(turn(f), f) <= Fraction(1, 2) + Fraction(1, 2 ** 44), f
    for e in range(-1074, 21):
        for f in (math.ldexp(1.0, e), math.ldexp(1.0, e) * (2 - 2.0 ** -52) if e > -1000 and e < 20 else 0.0):
            assert off(turn(f), f) <= Fraction(1, 2) + Fraction(1, 2 ** 44), f

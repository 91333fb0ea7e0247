"""The rotation's integer angles against exact fractions (CPU): compiled from the library's own source."""
import os
import random
import shutil
import subprocess
from fractions import Fraction

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
PI = Fraction("3.14159265358979323846264338327950288419716939937510582097494459230781640628620899")


@pytest.fixture(scope="module")
def turns(tmp_path_factory):
    cc = shutil.which("g++")
    if cc is None:
        pytest.skip("g++ not found")
    exe = str(tmp_path_factory.mktemp("turns") / "turns_check")
    subprocess.run([cc, "-std=c++17", "-O1", os.path.join(HERE, "turns_check.cpp"), "-o", exe], check=True)
    return lambda fs: [int(x) for x in subprocess.run([exe], input="\n".join(f.hex() for f in fs), capture_output=True, text=True,
                                                      check=True).stdout.split()]


def off(n, f):
    """units of 2^-64 of a turn between an integer angle and f / (2 pi), modulo a turn"""
    d = (n - Fraction(f) / (2 * PI) * 2 ** 64) % 2 ** 64
    return float(min(d, 2 ** 64 - d))


def test_frequencies_of_either_sign(turns):
    """Off by one unit at most: the product's high part is exact as a fraction, its low part is cut to units (less
    than one) and itself off by some 2^-20 of one."""
    rng = random.Random(1)
    fs = [b ** (-i / 64) for b in (1e4, 1e6, 1e12) for i in range(64)]
    fs += [0.0, 1e6, 7.25, 6.283185307179586, 1e-300, 5e-324, 2.0 ** -60] + [rng.uniform(0, 1e6) for _ in range(200)]
    fs += [2.0 ** rng.uniform(-70, 19) for _ in range(300)]
    for sign in (1, -1):
        got = turns([sign * f for f in fs])
        assert len(got) == len(fs)
        for n, f in zip(got, fs):
            assert 0 <= n < 2 ** 64 and off(n, sign * f) <= 1 + 2.0 ** -16, (sign * f, off(n, sign * f))


def test_the_other_way_round_is_the_negative_integer(turns):
    fs = [1e4 ** (-i / 64) for i in range(64)] + [123456.789, 0.0, -0.0]
    assert all((a + b) % 2 ** 64 == 0 for a, b in zip(turns(fs), turns([-f for f in fs])))

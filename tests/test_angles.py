"""CPU run of the angles of the rotation (csrc/angle.h) against exact fractions, at any position."""
import math
import os
import random
import struct
import subprocess
from fractions import Fraction

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
PI = Fraction(3141592653589793238462643383279502884197169399375105820974944592, 10 ** 63)          # (2^-206 off)

CODE = r"""
#include <cstdio>
#include "angle.h"
int main()
{
    float f;
    int p;
    while (std::scanf("%a %d", &f, &p) == 2) std::printf("%a\n", (double)cf::half_turns(f, p));
}
"""


def fp32(x):
    return struct.unpack("f", struct.pack("f", x))[0]


@pytest.fixture(scope="module")
def half_turns(tmp_path_factory):
    path = tmp_path_factory.mktemp("angle")
    (path / "angle.cpp").write_text(CODE)
    subprocess.run(["g++", "-O1", "-std=c++17", "-Wall", "-Werror", "-fsanitize=undefined", "-fno-sanitize-recover", "-I",
                    os.path.join(ROOT, "paper_2503_02356_amd", "csrc"), str(path / "angle.cpp"), "-o", str(path / "angle")], check=True)

    def run(calls):
        text = "\n".join(f"{f.hex() if math.isfinite(f) else f} {p}" for f, p in calls)
        r = subprocess.run([str(path / "angle")], input=text, capture_output=True, text=True)
        assert r.returncode == 0, r.stderr[-2000:]
        return [float.fromhex(x) for x in r.stdout.split()]
    return run


def off(got, f, p):
    """How far `got` half-turns are from f * p radians, whole turns aside, in half-turns."""
    left = (Fraction(got) - Fraction(f) * p / PI) % 2
    return float(min(left, 2 - left))


def cases():
    rng = random.Random(8)
    usual = [fp32(base ** (-i / 64)) for base in (1e4, 5e5, 1e6) for i in range(64)]
    frequencies = usual + [fp32(2 * math.pi), fp32(math.pi), 1.0, 0.5, -1.0, 100.0, 511.0, 1e-30, 0.0]
    positions = [0, 1, 2, 1000, 229375, 1 << 20, (1 << 28) + 1, (1 << 30) - 1, 1 << 30, (1 << 31) - 1]
    return [(f, p) for f in frequencies for p in positions] + [(fp32(math.exp(rng.uniform(-20, 6))), rng.randrange(1 << rng.randint(1, 31))) for _ in range(20000)]


def test_far_positions_are_as_exact_as_near_ones(half_turns):
    """One rounding to fp32 of a number of at most 1 and 2^-53 of the turns (the rounding by which whole turns are found, which may take the rest above 1, where half a
    step is 2^-24), two of numbers of about 1 to fp64 and parts of 2^-100 of the angle before."""
    calls = cases()
    for (f, p), got in zip(calls, half_turns(calls)):
        assert abs(got) <= 1 + abs(f) * p / 6 * 2.0 ** -52 + 2.0 ** -23
        bound = (2.0 ** -25 if abs(got) < 1 else 2.0 ** -24) + 2.0 ** -50
        assert off(got, f, p) <= bound, (f, p, off(got, f, p))


def test_near_positions_lose_no_bits(half_turns):
    """Below half a turn the result has the relative error of its rounding."""
    calls = [(f, p) for f, p in cases() if 0 < abs(f) * p < 3]
    assert len(calls) > 1000
    for (f, p), got in zip(calls, half_turns(calls)):
        assert off(got, f, p) <= abs(got) * (2.0 ** -24 + 2.0 ** -50)


def test_what_is_not_finite(half_turns):
    inf = float("inf")
    assert all(math.isnan(x) for x in half_turns([(inf, 0), (inf, 3), (-inf, 3), (float("nan"), 0), (float("nan"), 7)]))

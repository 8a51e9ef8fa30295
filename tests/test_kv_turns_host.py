"""Frequencies of rotary positions as 64-bit fractions of a turn (paper_2609_33224_gb300/csrc/kv_turns.h): off by no more
than the header's bound, frequencies of either sign alike."""
import os
import random
import subprocess
from fractions import Fraction

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2609_33224_gb300", "csrc")
TAU = 2 * Fraction("3.14159265358979323846264338327950288419716939937510582097494")

HARNESS = r"""
#include <cstdio>
#include "kv_turns.h"
int main() {
  double f;
  while (std::scanf("%la", &f) == 1) std::printf("%llu\n", (unsigned long long)pskv::turns_of(f));
}
"""


@pytest.fixture(scope="module")
def turns_of(tmp_path_factory):
    d = tmp_path_factory.mktemp("turns")
    src, exe = d / "t.cpp", d / "t"
    src.write_text(HARNESS)
    subprocess.run(["g++", "-std=c++17", "-O2", "-ffp-contract=off", "-I", CSRC, str(src), "-o", str(exe)], check=True)

    def run(fs):
        text = "".join(float(f).hex() + "\n" for f in fs)
        r = subprocess.run([str(exe)], input=text, capture_output=True, text=True, check=True)
        return [int(x) for x in r.stdout.split()]
    return run


def _frequencies():
    rng = random.Random(1)
    f = [10000.0 ** (-2 * i / 128) for i in range(64)] + [500000.0 ** (-2 * i / 128) / 8 for i in range(64)]
    f += [1e-5, 1e-6, 1e-12, 1e-19, 1e-20, 1e-300, 5e-324, 0.0, float(TAU), float(TAU) / 2, float(TAU) * (1 - 2.0 ** -53),
          7.0, 1e3, 1e9, 1e15, 2.0 ** 60]
    f += [rng.uniform(0, 1) * 2.0 ** rng.randint(-70, 40) for _ in range(2000)]
    return f


@pytest.mark.parametrize("sign", [1, -1])
def test_the_bound_holds_for_either_sign(turns_of, sign):
    """The angle of a position is off by at most |f| 2^-52 + 2^-62, whole turns aside: f / 2 pi is rounded twice (the
    quotient, and 2 pi itself), by 2^-53 of it each, and then to 2^-65 of a turn, which is 2^-62.3."""
    fs = [sign * f for f in _frequencies()]
    for f, got in zip(fs, turns_of(fs)):
        assert 0 <= got < 1 << 64
        d = Fraction(f) / TAU - Fraction(got, 1 << 64)
        d -= round(d)
        assert abs(d) * TAU <= abs(Fraction(f)) / 2 ** 52 + Fraction(1, 1 << 62), (f, float(d))


def test_a_negative_frequency_turns_the_other_way(turns_of):
    fs = _frequencies()
    for f, x, y in zip(fs, turns_of(fs), turns_of([-f for f in fs])):
        assert (x + y) % (1 << 64) == 0, f

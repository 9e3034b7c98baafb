"""A rate's turns per position (csrc/paged_turns.h) against decimals of 100 digits, compiled and run on the host."""
import decimal
import math
import os
import random
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2607_28979_gb300", "csrc")

PROGRAM = r"""
#include "paged_turns.h"
#include <cinttypes>
#include <cstdio>
int main(int argc, char** argv) {
  if (argc > 1) {   // rates of a base, as the default ones are made
    double base;
    int rot;
    while (std::scanf("%la %d", &base, &rot) == 2)
      for (int i = 0; i < rot / 2; ++i)
        std::printf("%" PRIu64 "\n", mot::turn_of(std::pow(static_cast<long double>(base), -2.0L * i / rot)));
    return 0;
  }
  double r;
  while (std::scanf("%la", &r) == 1) std::printf("%" PRIu64 "\n", mot::turn_of(r));
  return 0;
}
"""
PI = decimal.Decimal("3.14159265358979323846264338327950288419716939937510582097494459230781640628620899862803482534211706798214808651")


@pytest.fixture(scope="module")
def turns(tmp_path_factory):
    path = tmp_path_factory.mktemp("turns")
    src, exe = path / "turns.cpp", path / "turns"
    src.write_text(PROGRAM)
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-I", CSRC, str(src), "-o", str(exe)], check=True)

    def run(lines, *args):
        r = subprocess.run([str(exe), *args], input="\n".join(lines), capture_output=True, text=True, timeout=60, check=True)
        return [int(x) for x in r.stdout.split()]
    return run


def _off(got, rate):
    """How far `got` is from the rate's turns, in units of 2^-64, around the circle."""
    want = rate / (2 * PI)
    want = (want - want.to_integral_value(rounding=decimal.ROUND_FLOOR)) * 2 ** 64
    d = abs(want - got)
    return min(d, 2 ** 64 - d)


def _rates():
    rng = random.Random(7)
    rates = [0.0, -0.0, 1.0, 65536.0, 2 * math.pi, math.pi, 1e-300, 5e-324, 2.0 ** -62, math.nextafter(65536.0, 0), 52923.3, 16809.558]
    rates += [2.0 ** k for k in range(-70, 17)] + [k * math.pi for k in range(1, 20000, 997)]   # next to whole and half turns
    rates += [rng.uniform(0, 65536) for _ in range(2000)] + [2.0 ** rng.uniform(-68, 16) for _ in range(2000)]
    return rates + [-r for r in rates]


def test_turns_over_the_whole_range(turns):
    rates = _rates()
    got = turns([r.hex() for r in rates])
    assert len(got) == len(rates)
    with decimal.localcontext() as ctx:
        ctx.prec = 100
        # to the nearest: half a unit, and 2^-64 that is cut off (of a negative rate too)
        assert max(_off(g, decimal.Decimal(r)) for g, r in zip(got, rates)) <= decimal.Decimal("0.5") + decimal.Decimal(2) ** -62
    for r, g in zip(rates, got):
        if r == 0 or abs(r) < 2.0 ** -63:
            assert g == 0
    half = len(rates) // 2
    assert all((a + b) % 2 ** 64 == 0 for a, b in zip(got[:half], got[half:]))   # a rate and its negative cancel


def test_default_rates(turns):
    """base^(-2 i / rot): the power is off by 2 units of 2^-64 of itself at most (a long double has 64 bits at least), its
    turns by a sixth of that, and they are rounded to half a unit."""
    cases = [(1e4, 64), (1e6, 128), (5e5, 96), (1.0, 16), (10.5, 32), (1e30, 128)]
    got = turns([f"{float(b).hex()} {r}" for b, r in cases], "base")
    with decimal.localcontext() as ctx:
        ctx.prec = 100
        want = [decimal.Decimal(b) ** (decimal.Decimal(-2 * i) / r) for b, r in cases for i in range(r // 2)]
        assert len(got) == len(want)
        assert max(_off(g, w) for g, w in zip(got, want)) <= decimal.Decimal("0.9")

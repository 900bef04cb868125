"""Scales of orthogonalised updates (code of the device, run on the host; no GPU): bounds hold, images fill the range of halves, factors are finite
and undo one another, however small the matrix is beside eps and whatever the coefficients make of it."""
import math
import os
import subprocess

import numpy as np
import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
MUON = (3.4445, -4.775, 2.0315)


@pytest.fixture(scope="module")
def ask(tmp_path_factory):
    exe = str(tmp_path_factory.mktemp("scales") / "harness")
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", os.path.join(HERE, "update_scales_harness.cpp"), "-o", exe], check=True)

    def run(ratio, coefficients, out_scale=1.0):
        line = f"{ratio!r} {out_scale!r} {len(coefficients)} " + " ".join(repr(float(v)) for c in coefficients for v in c)
        got = [float(v) for v in subprocess.run([exe], input=line + "\n", capture_output=True, text=True, check=True).stdout.split()]
        names = ("gram", "square", "linear", "diagonal", "move", "scale", "most")
        return got[0], [dict(zip(names, got[1 + 7 * i:8 + 7 * i])) for i in range(len(coefficients))]
    return run


def scale(most):
    return 2.0 ** (15 - math.frexp(most)[1])     # (log2 of a number just below a power of two rounds up to its exponent)


@pytest.mark.parametrize("ratio, first", [(1.0, 1.0), (0.9, 1.0), (0.51, 1.0), (0.5, 0.5), (0.3, 0.5), (1.5, 1.0), (0.0, 1.0), (math.nan, 1.0), (2.0**-40, 2.0**-40),
                                          (1.1 * 2.0**-40, 2.0**-39), (1e-40, 2.0**-96)])
def test_the_first_bound_is_the_power_of_two_above(ask, ratio, first):
    assert ask(ratio, [])[0] == first


@pytest.mark.parametrize("coefficients", [[MUON] * 5, [(1.5, -0.5, 0.0)] * 3, [(0.0, 1.25, 0.0)], [(0.0, 0.0, 1.0)], [(1e-9, 0.0, 0.0), MUON], [(0.0, 0.0, 1e-12)] * 2,
                                          [(0.0, 0.0, 0.0), MUON], [(2.0, -1.5, 0.5)] * 12])
def test_scales_follow_the_bound_of_the_singular_values(ask, coefficients):
    for ratio in (1.0, 0.7, 1e-3, 1e-8, 1e-13, 1e-20, 1e-27):
        first, steps = ask(ratio, coefficients, 0.75)
        s = np.linspace(0, ratio, 2001)
        assert first >= ratio
        before = first
        for i, ((a, b, c), f) in enumerate(zip(coefficients, steps)):
            a, b, c = (float(np.float32(v)) for v in (a, b, c))
            factor = np.abs(a + before**2 * np.linspace(0, 1, 4001) ** 2 * (b + c * before**2 * np.linspace(0, 1, 4001) ** 2)).max()
            s = np.abs(s * (a + s**2 * (b + c * s**2)))
            assert s.max() <= f["most"] * (1 + 1e-12)
            assert all(math.isfinite(v) for v in f.values())
            x = scale(before)
            to = 1.0 if i + 1 == len(coefficients) else scale(f["most"])
            assert f["scale"] == (0.75 if i + 1 == len(coefficients) else 1.0)
            assert f["gram"] == pytest.approx(scale(before**2) / x**2, rel=1e-7)
            if factor > 0 and f["move"] > 0:
                # P fills the halves: its bound lies in 2^14 .. 2^15 (a grid of 4001 points misses a maximum by less than 1e-5 of it)
                p = 2.0 ** round(math.log2(to / (f["move"] * x)))
                assert 2.0**14 * (1 - 1e-12) <= factor * p * (1 + 1e-5) and factor * p < 2.0**15 * (1 + 1e-5)
                assert f["move"] == pytest.approx(to / (p * x), rel=1e-6)
                assert f["diagonal"] == pytest.approx(a * p, rel=1e-6)
                # what is left of a coefficient that falls out of fp32 is nothing beside the others: its share of P is below 2^-126 of the whole
                assert f["linear"] == pytest.approx(b * p / scale(before**2), rel=1e-6, abs=2.0**-126)
                assert f["square"] == pytest.approx(c * p / scale(before**2) ** 2, rel=1e-6, abs=2.0**-126)
            before = f["most"]


@pytest.mark.parametrize("coefficients", [(3.9, -3.9, 1e-20), (2.0, -1.5, 1e-30), (3.0, -3.0, -1e-17), (-3.9, 3.9, 1e-12), (0.5, 0.0, -1e-25), (0.0, 2.0, -1.5), (0.0, 0.0, 1.0)])
def test_bounds_hold_where_a_coefficient_is_nearly_zero(ask, coefficients):
    """Stationary points are roots of a + 3 b t + 5 c t^2, one of which a difference of nearly equal numbers would lose."""
    for ratio in (1.0, 0.8):
        first, steps = ask(ratio, [coefficients])
        s = np.linspace(0, first, 20001)
        a, b, c = (float(np.float32(v)) for v in coefficients)
        value = np.abs(s * (a + s**2 * (b + c * s**2))).max()
        # the grid's steps are 5e-5 and second derivatives below 30: it misses a maximum by less than 30 (5e-5)^2 / 8
        assert value <= steps[0]["most"] * (1 + 1e-12) and steps[0]["most"] <= value + 1e-8

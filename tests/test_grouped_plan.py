"""What the grouped products and orthogonalised updates refuse, and what they fill in (host code on its own; no GPU)."""
import os
import subprocess

import numpy as np
import pytest

HERE = os.path.dirname(os.path.abspath(__file__))


@pytest.fixture(scope="module")
def ask(tmp_path_factory):
    exe = str(tmp_path_factory.mktemp("grouped") / "harness")
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", os.path.join(HERE, "grouped_plan_harness.cpp"), "-o", exe], check=True)

    def run(*lines):
        out = subprocess.run([exe], input="\n".join(lines) + "\n", capture_output=True, text=True, check=True).stdout.splitlines()
        assert len(out) == len(lines)
        return out if len(out) > 1 else out[0]
    return run


def test_strides_left_at_zero_are_dense(ask):
    assert ask("p 1 1 4 100 30 50 0  0 0 0 0") == "ok 30 50 1500 50"
    assert ask("p 1 0 4 100 30 50 1  0 0 0 0") == "ok 30 30 1500 50"
    assert ask("p 1 0 4 100 30 50 0  32 56 0 64") == "ok 32 56 1680 64"
    assert ask("t 0 0 4 100 30 50  0 0 0 0") == "ok 30 50 50 1500"
    assert ask("t 2 0 4 100 30 50  0 0 64 0") == "ok 30 50 64 1920"


@pytest.mark.parametrize("line, why", [
    ("p 3 3 4 100 30 50 0 0 0 0 0", "type"), ("p -1 -1 4 100 30 50 0 0 0 0 0", "type"), ("p 1 2 4 100 30 50 0 0 0 0 0", "type"),
    ("p 0 1 4 100 30 50 0 0 0 0 0", "type"),
    ("p 1 1 0 100 30 50 0 0 0 0 0", "n_groups"), ("p 1 1 1025 100 30 50 0 0 0 0 0", "n_groups"),
    ("p 1 1 4 -1 30 50 0 0 0 0 0", "rows"), ("p 1 1 4 2147483393 30 50 0 0 0 0 0", "rows"),
    ("p 1 1 4 100 0 50 0 0 0 0 0", "k and n"), ("p 1 1 4 100 30 0 0 0 0 0 0", "k and n"), ("p 1 1 4 100 30 1048577 0 0 0 0 0", "k and n"),
    ("p 1 1 4 100 30 50 0 29 0 0 0", "leading"), ("p 1 1 4 100 30 50 0 0 49 0 0", "leading"), ("p 1 1 4 100 30 50 1 0 29 0 0", "leading"),
    ("p 1 1 4 100 30 50 0 0 0 0 49", "leading"), ("p 1 1 4 100 30 50 0 -30 0 0 0", "stride"), ("p 1 1 4 100 30 50 0 0 0 -1 0", "stride"),
    ("p 1 1 4 100 30 50 0 1099511627776 0 0 0", "stride"), ("p 1 1 4 100 30 50 0 0 0 0 0 1", "aligned"), ("p 0 0 4 100 30 50 0 0 0 0 0 2", "aligned"),
    ("t 1 1 4 100 30 50 0 0 49 0", "leading"), ("t 1 1 4 100 30 50 0 0 0 1499", "overlap"), ("t 1 1 4 100 0 50 0 0 0 0", "ka and nb"),
    ("o 1 2 1 8 8 1 0 1 1 1 1", "type"), ("o 1 1 0 8 8 1 0 1 1 1 1", "batch"), ("o 1 1 65536 8 8 1 0 1 1 1 1", "batch"),
    ("o 1 1 1 0 8 1 0 1 1 1 1", "rows and cols"), ("o 1 1 1 8 32769 1 0 1 1 1 1", "rows and cols"), ("o 1 1 1 8 8 65 0 1 1 0 0", "n_steps"),
    ("o 1 1 1 8 8 -1 0 1 1 0 0", "n_steps"), ("o 1 1 1 8 8 1 -1 1 1 0 0", "eps"), ("o 1 1 1 8 8 1 nan 1 1 0 0", "eps"),
    ("o 1 1 1 8 8 1 0 inf 1 0 0", "scale"),
    ("o 1 1 1 8 8 5 0 1 3 0 0", "grow"), ("o 1 1 1 8 8 1 0 1 0 0 2000", "grow")])
def test_refusals(ask, line, why):
    got = ask(line)
    assert not got.startswith("ok") and why in got, got


def test_accepted_edges(ask):
    for line in ("p 1 1 1024 2147483392 1048576 1048576 0 0 0 0 0", "p 0 0 1 0 1 1 1 0 0 0 0", "t 2 2 1 0 1 1 0 0 0 0", "p 2 2 4 100 30 50 0 0 0 0 0 2"):
        assert ask(line).startswith("ok"), line
    for line in ("o 0 0 65535 1 32768 0 0 1 0 0 0", "o 0 0 1 4096 4096 64 0 -1 3.4445 -4.775 2.0315", "o 2 0 1 8 8 64 0.5 0 1.875 -1.25 0.375",
                 "o 0 0 1 8 8 2 0 1 3.9 0 0"):
        assert ask(line) == "ok", line


def test_growth_is_the_maximum_over_the_interval(ask):
    rng = np.random.default_rng(0)
    for _ in range(300):
        most = float(10 ** rng.uniform(-2, 1))
        a, b, c = (float(v) for v in rng.normal(size=3) * rng.choice([0.0, 1.0, 5.0], size=3))
        value, factor = (float(v) for v in ask(f"g {most!r} {a!r} {b!r} {c!r}").split())
        s = np.linspace(0, most, 200001)
        f = np.abs(a + s**2 * (b + c * s**2))
        # between two points of the grid a polynomial of this size moves by less than its slope bound times the spacing, and at a maximum by its square
        assert value >= (s * f).max() * (1 - 1e-12) and value <= (s * f).max() * (1 + 1e-8) + 1e-12
        assert factor >= f.max() * (1 - 1e-12) and factor <= f.max() * (1 + 1e-8) + 1e-12

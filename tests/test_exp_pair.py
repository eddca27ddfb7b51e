"""The teacher's probabilities (csrc/exp_pair.hpp) on the host, with and without products and sums made one: to 2^-40, the bound that is derived there."""
import os
import subprocess

import pytest


@pytest.mark.parametrize("contract", ["off", "fast"])
def test_exponentials_of_pairs(contract, tmp_path):
    here = os.path.dirname(os.path.abspath(__file__))
    out = str(tmp_path / "exp_pair")
    subprocess.check_call(["g++", "-O2", "-std=c++17", "-Wall", "-march=native", "-ffp-contract=" + contract, "-o", out, os.path.join(here, "exp_pair.cpp")])
    done = subprocess.run([out], capture_output=True, text=True, timeout=300)
    assert done.returncode == 0, done.stdout

"""Every kernel that needs more dynamic LDS than a launch gets by itself has a bit of its own to remember that its limit was raised (no GPU)."""
import os
import subprocess

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(os.path.dirname(HERE), "paper_2303_13803_amd", "csrc")


@pytest.fixture(scope="module")
def bits(tmp_path_factory):
    program = str(tmp_path_factory.mktemp("lds_bits") / "lds_bits")
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Wextra", "-I", CSRC, "-o", program, os.path.join(HERE, "lds_bits.cpp")], check=True)
    return lambda rule: subprocess.run([program, rule], capture_output=True, text=True, timeout=120)


def test_no_two_kernels_share_a_bit(bits):
    done = bits("own")
    assert done.returncode == 0 and done.stdout.startswith("56 kernels"), done.stdout


def test_small_rounds_and_wide_fits_counted_from_the_same_bit(bits):
    done = bits("shared")
    assert done.returncode == 1 and " 4 bits taken twice" in done.stdout, done.stdout


def test_nothing_else_makes_such_bits():
    """Wherever a limit is raised its bit comes from the header."""
    for name in os.listdir(CSRC):
        text = open(os.path.join(CSRC, name)).read()
        assert text.count("hipFuncSetAttribute") == text.count("flag = lds_bit_"), name

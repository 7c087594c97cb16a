"""The error that csrc/rope_turn.h states for its sine and cosine, over a sweep of the arguments of a turn on the host: fmaf and the
fp32 products round there as they do on the device.

What the tests of the rotation allow a sine or cosine, 2^-22, follows from it: 1.73 x 2^-24 < 2^-23 here, and the angle is cut to 2^-32 of a
turn before (1.5e-9 radians, below 2^-29)."""
import os
import subprocess

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))


@pytest.fixture(scope="module")
def check(tmp_path_factory):
    exe = tmp_path_factory.mktemp("rope") / "rope_turn_check"
    # no contraction: the device code has none either where it matters (no sum but the fused ones)
    subprocess.run(["g++", "-O2", "-std=c++17", "-ffp-contract=off", "-o", str(exe), os.path.join(HERE, "native", "rope_turn_check.cpp")],
                   check=True)
    return lambda step: [float(x) for x in subprocess.run([str(exe), str(step)], capture_output=True, text=True, check=True).stdout.split()]


@pytest.mark.parametrize("step", [61, 64 * 1021 + 1])
def test_sine_and_cosine_are_off_by_no_more_than_stated(check, step):
    sine, cosine, polynomial_sine, polynomial_cosine = check(step)
    assert sine <= 1.73 and cosine <= 1.27                            # x 2^-24
    assert polynomial_sine <= 2.4e-8 and polynomial_cosine <= 6.7e-9

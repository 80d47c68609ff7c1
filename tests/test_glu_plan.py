"""Host arithmetic of the gated unit's products (csrc/glu_plan.h), built and run on the CPU."""
import os
import shutil
import subprocess

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))


@pytest.fixture(scope="module")
def program(tmp_path_factory):
    cxx = shutil.which("g++") or shutil.which("c++")
    if cxx is None:
        pytest.skip("no host compiler")
    exe = str(tmp_path_factory.mktemp("plan") / "glu_plan_host")
    subprocess.run([cxx, "-std=c++17", "-Wall", "-Werror", "-O1", "-o", exe, os.path.join(HERE, "glu_plan_host.cpp")], check=True,
                   timeout=300)
    return lambda *args: subprocess.run([exe, *map(str, args)], capture_output=True, text=True, check=True, timeout=60).stdout.split()


def test_no_whole_piece_ends_behind_its_operand(program):
    """Rows of 1 .. 40 elements, up to 300 values of k."""
    looked_at, *beyond = map(int, program("reads", 40, 300))
    assert looked_at > 10 ** 6 and not beyond, beyond


@pytest.mark.parametrize("k,step,a,b,whole", [
    (257, 64, 8, 8, 4), (256, 64, 8, 8, 4), (256, 64, 12, 8, 3), (257, 64, 12, 8, 4), (257, 32, 1, 1, 7), (263, 32, 1, 8, 8), (262, 32, 1, 8, 7),
    (64, 64, 0, 0, 1), (3, 32, 1, 0, 0), (0, 32, 5, 5, 0), (258, 32, 2, 0, 7), (259, 32, 0, 2, 8), (257, 32, 3, 0, 7), (258, 32, 0, 3, 8)])
def test_whole_steps(program, k, step, a, b, whole):
    assert program("steps", k, step, a, b) == [str(whole)]

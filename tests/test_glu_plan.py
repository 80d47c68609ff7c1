"""Host arithmetic of the gated unit's products (csrc/glu_plan.h), built and run on the CPU."""
import os
import random
import shutil
import subprocess

import pytest

from test_gpu_glu_plans import CASES

HERE = os.path.dirname(os.path.abspath(__file__))


@pytest.fixture(scope="module")
def program(tmp_path_factory):
    cxx = shutil.which("g++") or shutil.which("c++")
    if cxx is None:
        pytest.skip("no host compiler")
    exe = str(tmp_path_factory.mktemp("plan") / "glu_plan_host")
    subprocess.run([cxx, "-std=c++17", "-Wall", "-Werror", "-O1", "-o", exe, os.path.join(HERE, "glu_plan_host.cpp")], check=True,
                   timeout=300)
    return lambda *args: subprocess.run([exe, *map(str, args)], capture_output=True, text=True, check=True, timeout=60).stdout


def test_no_whole_piece_ends_behind_its_operand(program):
    """Rows of 1 .. 40 elements, up to 300 values of k."""
    looked_at, *beyond = map(int, program("reads", 40, 300).split())
    assert looked_at > 10 ** 6 and not beyond, beyond


@pytest.mark.parametrize("k,step,a,b,whole", [
    (257, 64, 8, 8, 4), (256, 64, 8, 8, 4), (256, 64, 12, 8, 3), (257, 64, 12, 8, 4), (257, 32, 1, 1, 7), (263, 32, 1, 8, 8), (262, 32, 1, 8, 7),
    (64, 64, 0, 0, 1), (3, 32, 1, 0, 0), (0, 32, 5, 5, 0), (258, 32, 2, 0, 7), (259, 32, 0, 2, 8), (257, 32, 3, 0, 7), (258, 32, 0, 3, 8)])
def test_whole_steps(program, k, step, a, b, whole):
    assert program("steps", k, step, a, b).split() == [str(whole)]


@pytest.mark.parametrize("T,H,F,dtype,forward,backward", CASES)
def test_which_tile_a_size_takes(program, T, H, F, dtype, forward, backward):
    """That each case of the GPU's tests is where it is meant to be."""
    assert program("plan", int(dtype == "f32"), 256, T, H, F) == f"{forward} | {backward} | fits\n"


def test_every_tile_has_a_case():
    """All that csrc/glu.hip can launch; in parts those that sizes of a training step are made in."""
    forward = {(c[3], c[4]) for c in CASES}
    assert forward >= {("bf16", t) for t in ("A256", "P256", "A128", "P128", "R128", "A64", "R64", "few 16", "few 64", "few 128")}
    assert forward >= {("bf16", t + "+") for t in ("A128", "R128", "A64", "R64")}
    assert forward >= {("f32", t) for t in ("R128", "R64", "R128+", "R64+")}
    backward = {(c[3], c[5].split(" ")[0]) for c in CASES}
    assert backward == {("bf16", t) for t in ("A256", "P256", "A128", "P128", "R128", "A64", "P64", "R64")} | {("f32", "R128"), ("f32", "R64")}
    assert {c[5].split(" ")[0] for c in CASES if "dx+" in c[5]} >= {"A256", "P256", "A128", "R128", "A64", "R64"}
    assert {c[5].split(" ")[0] for c in CASES if "dw+" in c[5]} >= {"A256", "A128", "R128", "A64", "R64"}


@pytest.mark.parametrize("cus", [256, 64, 304])
def test_parts_and_workspaces_of_any_size(program, cus):
    rng = random.Random(7)
    sizes = [(0, 0, 0), (1, 0, 1), (0, 8, 8), (8, 8, 0)]
    for _ in range(3000):
        T, H, F = (int(2 ** rng.uniform(0, top)) for top in (14, 13, 13.5))
        sizes.append((T, H // 8 * 8 + 8, F // 4 * 4 + 4) if rng.random() < 0.5 else (T, H, F))
    for f32 in (0, 1):
        lines = program("plan", f32, cus, *(n for s in sizes for n in s)).splitlines()
        assert len(lines) == len(sizes) and all(line.endswith("| fits") for line in lines)


@pytest.mark.parametrize("T,H,F,forward", [
    (24, 8192, 2048, "A64+"), (24, 8192, 5504, "few 64"), (64, 512, 2048, "A64"), (64, 776, 2500, "few 64"), (16, 8192, 2048, "A64+"),
    (16, 8192, 4096, "few 16"), (1, 1024, 4096, "few 16"), (64, 1024, 8192, "few 64"), (64, 4096, 9600, "few 128"),
    (65, 1024, 8192, "A64"), (8, 4096, 64, "A64+")])
def test_which_forward_few_rows_take(program, T, H, F, forward):
    """The faster one on either side of where it changes over, by the times in csrc/glu_plan.h."""
    assert program("plan", 0, 256, T, H, F).split(" | ")[0] == forward

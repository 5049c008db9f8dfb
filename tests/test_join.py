"""How a workgroup's wavefronts meet in shared memory (csrc/join.h), run on the CPU with the
wavefronts as far apart as barriers allow, in every order of rows with and without data."""
import os
import subprocess

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))


@pytest.fixture(scope="module")
def program(tmp_path_factory):
    out = str(tmp_path_factory.mktemp("join") / "join_waves")
    subprocess.run(["g++", "-std=c++17", "-O1", "-pthread", "-Wno-unknown-pragmas", "-o", out,
                    os.path.join(HERE, "join_waves.cpp")], check=True)
    return out


def test_joins_do_not_meet_each_other(program):
    r = subprocess.run([program], capture_output=True, text=True, timeout=120)
    assert r.returncode == 0 and r.stdout == "0 wrong\n"


def test_halves_that_go_by_rows_are_found_wrong(program):
    """A row without data has no barrier: two joins around it would share a half."""
    r = subprocess.run([program, "by_rows"], capture_output=True, text=True, timeout=120)
    assert r.returncode == 1 and int(r.stdout.split()[0]) > 0


def test_kernels_leave_the_halves_to_the_joins():
    """Nothing else in the kernels changes whose turn it is."""
    with open(os.path.join(HERE, "..", "paper_2601_17091_amd", "csrc", "rms_norm.hip")) as f:
        lines = [line.split("//")[0] for line in f]
    uses = [line.strip() for line in lines if "turn" in line.replace("return", "")]
    assert [u for u in uses if "join" not in u] == ["int turn = 0;"] * 2, uses

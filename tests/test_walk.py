"""The stages that a product of 8-bit rows asks for (csrc/walk.h), run on the CPU."""
import os
import subprocess

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))


@pytest.fixture(scope="module")
def program(tmp_path_factory):
    out = str(tmp_path_factory.mktemp("walk") / "walk")
    subprocess.run(["g++", "-std=c++17", "-O2", "-o", out, os.path.join(HERE, "walk.cpp")], check=True)
    return out


def test_every_stage_once_and_none_past_its_buffers(program):
    r = subprocess.run([program], capture_output=True, text=True, timeout=120)
    assert r.returncode == 0 and r.stdout == "0 wrong\n", r.stdout


def test_offsets_past_the_last_tile_are_found_wrong(program):
    """A buffer that holds nothing takes no offset that all lanes share."""
    r = subprocess.run([program, "as_if"], capture_output=True, text=True, timeout=120)
    assert r.returncode == 1 and int(r.stdout.split()[0]) > 0

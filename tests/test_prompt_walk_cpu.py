"""What a prompt's rows see, as the kernel walks it (csrc/wq4_seen.h), against the definition, on the CPU:
positions and lengths up to the largest that an int holds, windows and sinks of any size."""
import os
import subprocess

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(os.path.dirname(HERE), "paper_2412_15803_gb300", "csrc")


@pytest.fixture(scope="module")
def prompt_walk(tmp_path_factory):
    exe = str(tmp_path_factory.mktemp("walk") / "prompt_walk")
    subprocess.check_call(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-fsanitize=signed-integer-overflow,shift,bounds",
                           "-fsanitize-undefined-trap-on-error", "-I", CSRC, "-o", exe, os.path.join(HERE, "prompt_walk.cpp")])
    return exe


def run(exe, what, seed):
    r = subprocess.run([exe, what, "4000", str(seed)], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-2000:]


@pytest.mark.parametrize("seed", range(4))
def test_lookups_list_and_masks(prompt_walk, seed):
    run(prompt_walk, "walk", seed)


@pytest.mark.parametrize("seed", range(4))
def test_values_that_a_mask_hides(prompt_walk, seed):
    """Of what a copy brings into a tile, all that some row does not see is zeroed or looked at."""
    run(prompt_walk, "hidden", seed)

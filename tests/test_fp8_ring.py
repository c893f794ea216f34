"""The barriers of the 8-bit layer's kernels, in a model that runs their warps in many orders (tests/fp8_ring_model.cpp) with the kernels' own
rule of what a loader waits for at its end (csrc/fp8_ring.h): every wait ends, none too early, and nothing lands or arrives in shared memory
after the last warp has ended, also where a wait gave up."""
import os
import re
import subprocess

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
KERNELS = os.path.join(os.path.dirname(HERE), "paper_2410_09615_b200", "csrc", "fwd_fp8.cu")


@pytest.fixture(scope="module")
def model(tmp_path_factory):
    exe = str(tmp_path_factory.mktemp("ring") / "fp8_ring_model")
    subprocess.run(["g++", "-O2", "-std=c++17", "-Wall", "-Werror", os.path.join(HERE, "fp8_ring_model.cpp"), "-o", exe], check=True)
    return exe


# places, buffers, groups of a buffer, groups, tiles
SMALL = [(5, 2, 4, 1, 1), (5, 2, 4, 4, 1), (5, 2, 4, 5, 1), (5, 2, 4, 19, 1), (4, 2, 2, 16, 1), (7, 2, 2, 9, 1), (4, 2, 1, 13, 1)]
TOKENS = [(5, 2, 1, 1, 1), (5, 2, 1, 7, 3), (5, 4, 1, 4, 4), (6, 4, 1, 3, 5), (8, 4, 1, 9, 2), (2, 2, 1, 1, 9)]


@pytest.mark.parametrize("withheld", [-1, 0, 3])
@pytest.mark.parametrize("pair, shape", [(0, s) for s in SMALL + TOKENS] + [(1, s) for s in TOKENS])
def test_nothing_is_in_flight_at_the_end(model, pair, shape, withheld):
    groups = shape[3] * shape[4]
    out = subprocess.run([model, str(pair), *map(str, shape), str(withheld if withheld < groups else groups - 1), "400"], capture_output=True, text=True, timeout=120)
    assert out.stdout == "ok\n", out.stdout


def test_both_kernels_wait_by_that_rule():
    """Each kernel's loaders end in it, behind their requests, which end where a wait gives up."""
    text = re.sub(r"//[^\n]*", "", open(KERNELS).read())
    bodies = dict(zip(("fp8_small_kernel", "fp8_tokens_kernel"), re.split(r"__global__", text)[1:3]))
    assert "ring_tail(" in text
    for name, body in bodies.items():
        assert name in body
        loader, rest = body[body.index("auto request" if "small" in name else "const bool tokens"):].split("drain(empty,", 1)
        assert "tma_tile(" in loader and "tma_tile(" not in rest and rest.count("settle(abort_flag)") == 1, name
        assert len(re.findall(r"if \([^;]*\bwarp_wait\([^;]*break;", loader)) == loader.count("warp_wait(") == 1, name

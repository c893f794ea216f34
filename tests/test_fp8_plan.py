"""The host's choice of a kernel for the 8-bit layer, over all of its range: one that takes the call, clusters that are resident, tokens and
rows covered."""
import os
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_plans(tmp_path):
    exe = tmp_path / "fp8_plan"
    subprocess.check_call(["g++", "-O1", "-std=c++17", "-Wall", "-Werror", "-I", os.path.join(ROOT, "paper_2410_09615_b200", "csrc"),
                           os.path.join(ROOT, "tests", "fp8_plan.cpp"), "-o", str(exe)])
    assert subprocess.check_output([str(exe)], text=True).strip() == "ok"

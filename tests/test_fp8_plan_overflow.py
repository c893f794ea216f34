"""The 8-bit layer's plans over the whole range of sizes, compiled so that an integer that overflows, or a number that does not fit the type it
is turned into, ends the program."""
import os
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_no_arithmetic_of_a_plan_overflows(tmp_path):
    exe = tmp_path / "fp8_plan"
    subprocess.check_call(["g++", "-O1", "-std=c++17", "-Wall", "-Werror", "-fsanitize=undefined,float-cast-overflow", "-fno-sanitize-recover=all",
                           "-I", os.path.join(ROOT, "paper_2410_09615_b200", "csrc"), os.path.join(ROOT, "tests", "fp8_plan.cpp"), "-o", str(exe)])
    out = subprocess.run([str(exe)], capture_output=True, text=True)
    assert out.returncode == 0 and out.stdout.strip() == "ok", out.stderr

"""The plan of the residual norms' registers for every width, compiled for the host."""
import os
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_registers_hold_every_row_they_are_planned_for(tmp_path):
    exe = str(tmp_path / "row_plan")
    src = os.path.join(ROOT, "tests", "row_plan_driver.cpp")
    subprocess.run(["g++", "-O1", "-std=c++17", "-Wall", "-Werror", "-I" + os.path.join(ROOT, "paper_2004_09910_amd", "csrc"),
                    src, "-o", exe], check=True, timeout=120)
    r = subprocess.run([exe], capture_output=True, text=True, timeout=120)
    assert r.returncode == 0, r.stdout

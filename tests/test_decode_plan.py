"""How the decode side lays out its work, checked on the host: every part and column has a workgroup, LDS and scratch hold what is put there, and scratch
for a bound on the lengths serves every lower one."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.skipif(shutil.which("g++") is None, reason="needs g++")
def test_plans(tmp_path):
    exe = tmp_path / "decode_plan_driver"
    subprocess.check_call(["g++", "-O2", "-std=c++17", "-Wall", "-Wextra", "-Werror",
                           "-I", os.path.join(ROOT, "paper_2406_11674_amd", "csrc"),
                           os.path.join(ROOT, "tests", "decode_plan_driver.cpp"), "-o", str(exe)])
    proc = subprocess.run([str(exe)], stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True, timeout=120)
    assert proc.returncode == 0, proc.stdout
    assert proc.stdout.startswith("ok"), proc.stdout

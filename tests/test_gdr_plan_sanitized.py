"""The planner of the gated delta rule (pgf_gdr_plan.cpp, plain C++) under
AddressSanitizer and UndefinedBehaviorSanitizer (no GPU)."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.skipif(shutil.which("g++") is None, reason="no g++")
def test_gdr_planner_under_sanitizers(tmp_path):
    exe = str(tmp_path / "gdr_plan_driver")
    subprocess.run(["g++", "-std=c++17", "-O1", "-fsanitize=address,undefined", "-fno-sanitize-recover=all", "-g", "-o",
                    exe, os.path.join(ROOT, "tests", "sanitize", "gdr_plan_driver.cpp"),
                    os.path.join(ROOT, "paper_2512_23068_amd", "csrc", "pgf_gdr_plan.cpp")], check=True)
    r = subprocess.run([exe], capture_output=True, text=True, timeout=300)
    print(r.stdout, r.stderr)
    assert r.returncode == 0, r.stdout + r.stderr
    assert " 0 failures" in r.stdout and "ERROR" not in r.stderr and "runtime error" not in r.stderr

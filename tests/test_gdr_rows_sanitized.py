"""Rows of the gated delta rule's arrays as its kernels take them: the host's part
(plain C++) under AddressSanitizer and UndefinedBehaviorSanitizer (no GPU)."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
pytestmark = pytest.mark.skipif(shutil.which("g++") is None, reason="no g++")


@pytest.fixture(scope="module")
def driver(tmp_path_factory):
    exe = str(tmp_path_factory.mktemp("rows") / "gdr_rows_driver")
    subprocess.run(["g++", "-std=c++17", "-O1", "-fsanitize=address,undefined", "-fno-sanitize-recover=all", "-g", "-o",
                    exe, os.path.join(ROOT, "tests", "sanitize", "gdr_rows_driver.cpp"),
                    os.path.join(ROOT, "paper_2512_23068_amd", "csrc", "pgf_gdr_plan.cpp")], check=True)
    return exe


def run(driver, what):
    r = subprocess.run([driver, what], capture_output=True, text=True, timeout=300)
    print(r.stdout, r.stderr)
    assert r.returncode == 0, r.stdout + r.stderr
    assert " 0 failures" in r.stdout and "ERROR" not in r.stderr and "runtime error" not in r.stderr


def test_rows_of_one_step(driver):
    """A single step's rows end behind it, also where its step stride is zero."""
    run(driver, "one")


def test_rows_of_outputs_lie_apart(driver):
    """Outputs whose rows overlap are refused, others are taken in any order."""
    run(driver, "apart")


def test_parts_of_one_array(driver):
    """Parts of one array's rows are taken, head by head too."""
    run(driver, "parts")

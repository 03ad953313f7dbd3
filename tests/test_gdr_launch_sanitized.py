"""Launch sizes of the gated delta rule: the host's part (plain C++) under
AddressSanitizer and UndefinedBehaviorSanitizer, and the planning calls (no GPU)."""
import os
import shutil
import subprocess

import pytest

from tests.test_gdr_abi import OK, UNSUPPORTED, gdr, plan

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.skipif(shutil.which("g++") is None, reason="no g++")
def test_launches_under_sanitizers(tmp_path):
    exe = str(tmp_path / "gdr_launch_driver")
    subprocess.run(["g++", "-std=c++17", "-O1", "-fsanitize=address,undefined", "-fno-sanitize-recover=all", "-g", "-o",
                    exe, os.path.join(ROOT, "tests", "sanitize", "gdr_launch_driver.cpp"),
                    os.path.join(ROOT, "paper_2512_23068_amd", "csrc", "pgf_gdr_plan.cpp")], check=True)
    r = subprocess.run([exe], capture_output=True, text=True, timeout=300)
    print(r.stdout, r.stderr)
    assert r.returncode == 0, r.stdout + r.stderr
    assert " 0 failures" in r.stdout and "ERROR" not in r.stderr and "runtime error" not in r.stderr


@pytest.mark.parametrize("kw,code", [
    # one block of 256 threads a state of 64 columns; 2^24 of them are 2^32 threads
    (dict(batch=(1 << 20) - 1, d_value=64), OK), (dict(batch=1 << 20, d_value=64), UNSUPPORTED),
    # the gradients' outer products: 512 threads a head and 64 steps
    (dict(batch=1 << 19, d_value=8), OK), (dict(batch=1 << 19, d_value=8, grads=1), UNSUPPORTED),
    (dict(batch=(1 << 19) - 1, d_value=8, grads=1), OK),
    # rows of no sequence: 64 a block
    (dict(batch=1, n_seqs=2, key_heads=1, value_heads=1, d_value=8, seqlen=(1 << 30) - 64, clear_rest=1), OK),
    (dict(batch=1, n_seqs=2, key_heads=1, value_heads=1, d_value=8, seqlen=1 << 30, clear_rest=1), UNSUPPORTED)])
def test_largest_launches(kw, code):
    assert plan(gdr(**{**dict(key_heads=16, value_heads=16, seqlen=1, d_key=8), **kw}))[0] == code

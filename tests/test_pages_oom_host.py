"""The allocator's calls when host memory runs out (CPU)."""

import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.skipif(shutil.which("g++") is None, reason="g++ not available")
def test_a_call_that_runs_out_of_memory_changes_nothing(tmp_path):
    csrc, exe = os.path.join(ROOT, "paper_2504_03775_amd", "csrc"), str(tmp_path / "oom_check")
    subprocess.run(["g++", "-std=c++17", "-O1", "-g", "-fsanitize=address,undefined",
                    "-fno-sanitize-recover=all", "-I", os.path.join(ROOT, "include"), "-I", csrc,
                    os.path.join(ROOT, "tests", "native", "pages_oom_check.cpp"),
                    os.path.join(csrc, "flowkv_alloc.cpp"), os.path.join(csrc, "flowkv_status.cpp"),
                    "-o", exe], check=True, capture_output=True, timeout=300)
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=1:verify_asan_link_order=0")
    r = subprocess.run([exe], capture_output=True, text=True, timeout=300, env=env)
    assert r.returncode == 0 and "failures ok" in r.stdout, r.stdout + r.stderr
    assert int(r.stdout.split()[0]) > 0          # (some allocations did fail)

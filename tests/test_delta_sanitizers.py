"""The delta rule's and the norm's host plans under the address and undefined-behaviour
sanitizers (CPU only): tests/sanitize/delta_plan_check.cpp with host_plan.cpp walks
configurations up to the ends of their integer types, and random ones, through the
checks, workspace sizes and segment plans that every entry point runs before it enqueues
anything."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_delta_plans_under_sanitizers(tmp_path):
    if shutil.which("g++") is None:
        pytest.skip("g++ not available")
    exe = str(tmp_path / "driver")
    r = subprocess.run(["g++", "-std=c++17", "-O1", "-g", "-fsanitize=address,undefined",
                        "-fno-sanitize-recover=all", "-fno-omit-frame-pointer",
                        os.path.join(ROOT, "tests/sanitize/delta_plan_check.cpp"),
                        os.path.join(ROOT, "paper_2609_12399_amd/csrc/host_plan.cpp"),
                        "-o", exe], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    r = subprocess.run([exe], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, f"{r.stdout}\n{r.stderr[-4000:]}"
    assert "delta plan checks: ok" in r.stdout

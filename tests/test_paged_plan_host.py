"""Host checks of paged attention (no GPU), compiled against the sources: how its
launches are planned (tests/native/paged_plan_check.cpp), and what in place means
(tests/native/paged_in_place_check.cpp)."""
import os
import shutil
import subprocess

import pytest

from tests.test_schedule_host import _build_and_run

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_plans_of_attention(tmp_path):
    hipcc = shutil.which("hipcc") or "/opt/rocm/bin/hipcc"
    if not os.path.exists(hipcc):
        pytest.skip("hipcc not found")
    exe = str(tmp_path / "paged_plan_check")
    cmd = [hipcc, "-x", "hip", "--offload-arch=gfx950", "-std=c++17", "-O1", "-fwrapv",
           "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
           "-I", os.path.join(ROOT, "include"), "-o", exe,
           os.path.join(ROOT, "tests", "native", "paged_plan_check.cpp")]
    r = subprocess.run(cmd, capture_output=True, text=True, timeout=600)
    assert r.returncode == 0, r.stderr[-2000:]
    out = subprocess.run([exe], capture_output=True, text=True, timeout=300)
    assert out.returncode == 0, out.stdout + out.stderr
    assert int(out.stdout.split()[1]) > 8000


def test_in_place_means_the_same_rows(tmp_path):
    assert _build_and_run(tmp_path, "paged_in_place_check") == 12

"""Launches of 2^32 threads or more are refused by the calls around a quantised cache, on the CPU (tests/host_launch_limits.hip)."""
import os
import subprocess

import pytest

from paper_2512_07090_amd import build as hip_build

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.skipif(not os.path.exists(hip_build.HIPCC), reason="needs hipcc")
def test_launches_that_are_too_large_are_refused(tmp_path):
    if not os.path.exists(hip_build.LIB):
        hip_build.build()
    exe = str(tmp_path / "launch_limits")
    pkg = os.path.dirname(hip_build.LIB)
    subprocess.check_call([hip_build.HIPCC, *hip_build.FLAGS, os.path.join(ROOT, "tests", "host_launch_limits.hip"), "-L" + pkg,
                           "-l:" + os.path.basename(hip_build.LIB), "-Wl,-rpath," + pkg, "-o", exe], stderr=subprocess.DEVNULL)
    r = subprocess.run([exe], capture_output=True, text=True, timeout=120)
    assert r.returncode == 0, r.stdout + r.stderr
    assert "launch limits: 0 failures" in r.stdout

"""What the calls around a quantised cache refuse, and its sizes, on the CPU: tests/host_cache_refusals.hip holds the library's
host code and is built with AddressSanitizer and UndefinedBehaviorSanitizer on the host pass only."""
import os
import shutil
import subprocess

import pytest

from paper_2512_07090_amd import build as hip_build

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.skipif(not os.path.exists(hip_build.HIPCC) or shutil.which("g++") is None, reason="needs hipcc and g++")
def test_refusals_and_sizes_without_a_gpu(tmp_path):
    if not os.path.exists(hip_build.LIB):
        hip_build.build()
    san = ["-Xarch_host", "-fsanitize=address", "-Xarch_host", "-fsanitize=undefined"]
    exe = str(tmp_path / "cache_refusals")
    pkg = os.path.dirname(hip_build.LIB)
    # the kernels' launchers come from the in-tree library; the entry points of this build win
    subprocess.check_call([hip_build.HIPCC, *hip_build.FLAGS, "-O1", "-g", *san,
                           os.path.join(ROOT, "tests", "host_cache_refusals.hip"), "-L" + pkg,
                           "-l:" + os.path.basename(hip_build.LIB), "-Wl,-rpath," + pkg, "-o", exe],
                          stderr=subprocess.DEVNULL)
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=0")   # the HIP runtime keeps process-lifetime allocations
    r = subprocess.run([exe], capture_output=True, text=True, env=env, timeout=120)
    assert r.returncode == 0, r.stdout + r.stderr
    assert "runtime error" not in r.stderr and "ERROR: AddressSanitizer" not in r.stderr, r.stderr
    assert "cache refusals: 0 failures" in r.stdout

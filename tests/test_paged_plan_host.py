"""The paged attention's host-side plan (grid and workspace) built with g++ under
AddressSanitizer and UndefinedBehaviorSanitizer and held against every choice
that the device may make from the lengths, over drawn shapes, lengths and
chunks. CPU only."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
SRC = [os.path.join(ROOT, "tests", "native", "paged_plan_check.cpp"),
       os.path.join(ROOT, "paper_2302_01318_amd", "csrc", "plan.cpp")]


@pytest.mark.skipif(shutil.which("g++") is None, reason="g++ not available")
def test_paged_plan_holds_what_the_device_may_choose(tmp_path):
    exe = str(tmp_path / "paged_plan_check")
    flags = ["-std=c++17", "-O1", "-g", "-Wall", "-fno-omit-frame-pointer",
             "-fsanitize=address,undefined", "-fno-sanitize-recover=all"]
    r = subprocess.run(["g++"] + flags + ["-I" + os.path.join(ROOT, "include")] + SRC + ["-o", exe],
                       capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-4000:]
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=1:abort_on_error=0",
               UBSAN_OPTIONS="print_stacktrace=1:halt_on_error=1")
    env.pop("LD_PRELOAD", None)
    r = subprocess.run([exe], capture_output=True, text=True, env=env, timeout=600)
    assert r.returncode == 0, (r.stdout + r.stderr)[-4000:]
    assert "paged plan check ok" in r.stdout

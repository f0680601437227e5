"""The 8-bit cache's index arithmetic (csrc/kvq_layout.h: the order of a
unit's bytes, pages outside the table or the pool, the pages of a run, the
slots a node sees) under AddressSanitizer and UndefinedBehaviorSanitizer, in a
host-only build of the header that the kernels include."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.skipif(shutil.which("g++") is None, reason="needs g++")
def test_kvq_layout_under_sanitizers(tmp_path):
    exe = tmp_path / "kvq_layout_test"
    src = os.path.join(ROOT, "tests", "native", "kvq_layout_test.cpp")
    inc = os.path.join(ROOT, "paper_2412_10418_amd", "csrc")
    cmd = ["g++", "-std=c++17", "-O1", "-g", "-fno-omit-frame-pointer", "-fsanitize=address,undefined",
           "-fno-sanitize-recover=all", "-I", inc, src, "-o", str(exe)]
    r = subprocess.run(cmd, capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=1:verify_asan_link_order=0",
               UBSAN_OPTIONS="print_stacktrace=1")
    r = subprocess.run([str(exe)], capture_output=True, text=True, env=env, timeout=120)
    assert r.returncode == 0, r.stdout + r.stderr
    assert "kvq layout: ok" in r.stdout

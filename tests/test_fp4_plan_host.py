"""The plan of the attention over the 4-bit cache (csrc/tree_plan.h) in a host-only build under AddressSanitizer and
UndefinedBehaviorSanitizer: the shapes of fp4_cases.py take the kernels that they are there for, all of them are taken at
every head dimension that has them to itself, and the kernels' assumptions hold over drawn sizes."""
import os
import shutil
import subprocess

import pytest

from fp4_cases import ALL, MANY_PAGES
from tree_cases import KINDS

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.skipif(shutil.which("g++") is None, reason="needs g++")
def test_shapes_take_the_kernels_that_they_test(tmp_path):
    exe = tmp_path / "fp4_plan_test"
    cmd = ["g++", "-std=c++17", "-O1", "-g", "-fno-omit-frame-pointer", "-fsanitize=address,undefined",
           "-fno-sanitize-recover=all", "-I", os.path.join(ROOT, "paper_2412_10418_amd", "csrc"),
           os.path.join(ROOT, "tests", "native", "fp4_plan_test.cpp"), "-o", str(exe)]
    r = subprocess.run(cmd, capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    asked = [(c, k) for c in ALL + MANY_PAGES for k in KINDS]
    lines = "".join(f"{c.B} {c.n} {c.H} {c.heads} {c.hd} {c.longest} {KINDS.index(k)}\n" for c, k in asked)
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=1:verify_asan_link_order=0", UBSAN_OPTIONS="print_stacktrace=1")
    r = subprocess.run([str(exe)], input=lines, capture_output=True, text=True, env=env, timeout=120)
    assert r.returncode == 0, r.stdout + r.stderr
    got = r.stdout.split()
    for (c, k), kernel in zip(asked, got):
        assert kernel == c.kernel(k, "mxfp4"), (c.name, k, kernel)
    assert got[len(asked):] == ["fp4", "plan:", "ok"]
    taken = {(kernel, k, c.hd) for (c, k), kernel in zip(asked, got)}
    for k in KINDS:
        for kernel in ("few1", "few2", "many", "few1+split", "few2+split", "many+split", "wide+split", "paired"):
            assert (kernel, k, 128) in taken, (kernel, k)
        for hd in (32, 64):
            assert {("many", k, hd), ("paired", k, hd), ("wide+split", k, hd)} <= taken
    assert {("wide", "bf16", hd) for hd in (32, 64, 128)} <= taken

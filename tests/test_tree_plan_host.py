"""The tree attention's plan (csrc/tree_plan.h) in a host-only build under AddressSanitizer and
UndefinedBehaviorSanitizer: the shapes of tree_cases.py take the kernels that they are there for, all of them are
taken, and the kernels' assumptions hold over drawn sizes."""
import os
import shutil
import subprocess

import pytest

from tree_cases import ALL, FMTS, KINDS

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.skipif(shutil.which("g++") is None, reason="needs g++")
def test_shapes_take_the_kernels_that_they_test(tmp_path):
    exe = tmp_path / "tree_plan_test"
    cmd = ["g++", "-std=c++17", "-O1", "-g", "-fno-omit-frame-pointer", "-fsanitize=address,undefined",
           "-fno-sanitize-recover=all", "-I", os.path.join(ROOT, "paper_2412_10418_amd", "csrc"),
           os.path.join(ROOT, "tests", "native", "tree_plan_test.cpp"), "-o", str(exe)]
    r = subprocess.run(cmd, capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    asked = [(c, k, f) for c in ALL for k in KINDS for f in FMTS]
    lines = "".join(f"{c.B} {c.n} {c.H} {c.heads} {c.hd} {c.longest} {KINDS.index(k)} {FMTS.index(f)}\n" for c, k, f in asked)
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=1:verify_asan_link_order=0", UBSAN_OPTIONS="print_stacktrace=1")
    r = subprocess.run([str(exe)], input=lines, capture_output=True, text=True, env=env, timeout=120)
    assert r.returncode == 0, r.stdout + r.stderr
    got = r.stdout.split()
    taken = set()
    for (c, k, f), kernel in zip(asked, got):
        assert kernel == c.kernel(k, f), (c.name, k, f, kernel)
        if c.hd == 128:
            taken.add((kernel, k, f))
    assert got[len(asked):] == ["tree", "plan:", "ok"]
    # every kernel that heads of 128 have, whole and (but for four waves a SIMD, which fill the chip) over split keys
    for k in KINDS:
        for f in FMTS:
            want = {"few1", "few2", "many3", "few1+split", "few2+split", "many3+split"}
            if (k, f) != ("f32", "e4m3"):
                want |= {"wide", "wide+split"}
            if k == "bf16" or f == "e4m3":
                want.add("many4")
            assert want <= {kernel for kernel, *types in taken if types == [k, f]}, (k, f)

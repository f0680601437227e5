"""The pages' calls without a GPU: their plans under AddressSanitizer and UndefinedBehaviorSanitizer (csrc/pages.h), and their
refusals, made on the host before anything is launched, on pointers that are never followed."""
import ctypes as C
import os
import shutil
import subprocess

import pytest
import torch

from test_tree_ops_host import P, _cache

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
TABLE, REFS, A, B_, OUT, WS = (P + 0x10000 * i for i in range(1, 7))


@pytest.mark.skipif(shutil.which("g++") is None, reason="needs g++")
def test_pages_plan_under_sanitizers(tmp_path):
    exe = tmp_path / "pages_plan_test"
    src = os.path.join(ROOT, "tests", "native", "pages_plan_test.cpp")
    inc = os.path.join(ROOT, "paper_2412_10418_amd", "csrc")
    cmd = ["g++", "-std=c++17", "-O1", "-g", "-fno-omit-frame-pointer", "-fsanitize=address,undefined",
           "-fno-sanitize-recover=all", "-I", inc, src, "-o", str(exe)]
    r = subprocess.run(cmd, capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=1:verify_asan_link_order=0",
               UBSAN_OPTIONS="print_stacktrace=1")
    r = subprocess.run([str(exe)], capture_output=True, text=True, env=env, timeout=120)
    assert r.returncode == 0, r.stdout + r.stderr
    assert "pages plan: ok" in r.stdout


def _lib():
    from paper_2412_10418_amd import binding as bd
    return bd.lib()


def _ref(c):
    return C.addressof(c) if c else None


def _fork(c, table=TABLE, refs=REFS, parents=A, ws=None, n=0):
    return _lib().cdsl_op_pages_fork(_ref(c), table, refs, parents, ws, n, None)


def _reserve(c, table=TABLE, refs=REFS, lens=A, count=B_, most=4, got=OUT, ws=WS, n=1 << 20):
    return _lib().cdsl_op_pages_reserve(_ref(c), table, refs, lens, count, most, got, ws, n, None)


def _free(c, table=TABLE, refs=REFS, lens=A):
    return _lib().cdsl_op_pages_free(_ref(c), table, refs, lens, None)


def _compact(c, table=TABLE, refs=REFS, used=OUT, ws=WS, n=1 << 20):
    return _lib().cdsl_op_pages_compact(_ref(c), table, refs, used, ws, n, None)


def _copy(c, to=None, src=A, dst=B_, n=3):
    return _lib().cdsl_op_pages_copy(_ref(c), src, _ref(to or c), dst, n, None)


CALLS = (_fork, _reserve, _free, _compact)


@pytest.mark.parametrize("kw", [dict(pool=None), dict(table=None), dict(n_layers=0), dict(pages=0), dict(n_kv_heads=0), dict(head_dim=48),
                                dict(batch=-1), dict(table_stride=0), dict(format=2), dict(pool=P + 8)], ids=str)
def test_bad_caches_are_refused_by_every_call(kw):
    from paper_2412_10418_amd.binding import CDSL_EINVAL
    for f in CALLS + (_copy,):
        assert f(_cache(**kw)) == CDSL_EINVAL, f.__name__
        assert f(None) == CDSL_EINVAL
    assert _copy(_cache(), _cache(**kw)) == CDSL_EINVAL


def test_null_and_overlapping_arrays():
    from paper_2412_10418_amd.binding import CDSL_EINVAL
    c = _cache()       # 3 prompts x 5 entries, 8 pages
    for f in CALLS:
        assert f(c, table=None) == f(c, refs=None) == CDSL_EINVAL, f.__name__
        assert f(c, refs=TABLE) == f(c, refs=TABLE + 56) == f(c, table=REFS + 28) == CDSL_EINVAL, f.__name__
    for at in (TABLE, TABLE + 56, REFS + 28, REFS - 8, None):
        assert _fork(c, parents=at) == _free(c, lens=at) == CDSL_EINVAL
        assert _reserve(c, lens=at) == _reserve(c, count=at) == _reserve(c, got=at) == CDSL_EINVAL
    assert _reserve(c, got=A) == _reserve(c, got=A + 8) == _reserve(c, got=B_ - 8) == CDSL_EINVAL
    assert _compact(c, used=None) == _compact(c, used=TABLE) == _compact(c, used=REFS + 28) == CDSL_EINVAL
    assert _reserve(c, most=-1) == CDSL_EINVAL
    assert _copy(c, src=None) == _copy(c, dst=None) == _copy(c, n=-1) == CDSL_EINVAL


def test_workspaces_apart_from_the_arrays():
    from paper_2412_10418_amd.binding import CDSL_EINVAL
    c, big, n = _cache(), _cache(batch=513, table_stride=9), 1 << 15
    for at in (TABLE, TABLE + 48, REFS, REFS - 16, A, B_, OUT):
        assert _reserve(c, ws=at, n=n) == CDSL_EINVAL, hex(at)
    for at in (TABLE, TABLE + 48, REFS, REFS - 16, OUT):
        assert _compact(c, ws=at, n=n) == CDSL_EINVAL, hex(at)
    for at in (TABLE, TABLE + 48, REFS, REFS - 16, A):
        assert _fork(big, ws=at, n=n) == CDSL_EINVAL, hex(at)


def test_pools_that_overlap():
    """Layers of pools that begin together but hold other numbers of pages, or a pool that begins inside another."""
    from paper_2412_10418_amd.binding import CDSL_EINVAL, CDSL_OK
    c = _cache()
    assert _copy(c, _cache(pages=9)) == _copy(c, _cache(pool=P + 16)) == _copy(_cache(pool=P + 16), c) == CDSL_EINVAL
    assert _copy(c, c, n=0) == _copy(c, _cache(pool=P + (1 << 30)), n=0) == CDSL_OK


def test_workspaces():
    from paper_2412_10418_amd.binding import CDSL_EINVAL
    L, c = _lib(), _cache()
    need = L.cdsl_op_pages_workspace(3, 5, 8, 4)
    assert 0 < need < 1000
    for ws, n in ((None, 1 << 20), (WS, 4), (WS + 4, 1 << 20)):
        assert _reserve(c, ws=ws, n=n) == _compact(c, ws=ws, n=n) == CDSL_EINVAL
    big = _cache(batch=513, table_stride=9)
    for ws, n in ((None, 0), (WS, 513 * 9 * 4 - 1), (WS + 8, 1 << 20)):
        assert _fork(big, ws=ws, n=n) == CDSL_EINVAL
    assert L.cdsl_op_pages_workspace(513, 9, 8, 0) >= 513 * 9 * 4
    assert L.cdsl_op_pages_workspace(0, 1, 100, 0) >= 4 * 100           # compacting needs no prompts
    for bad in ((-1, 5, 8, 4), (65536, 5, 8, 4), (3, 0, 8, 4), (3, 1 << 26, 8, 4), (3, 5, 0, 4), (3, 5, (1 << 30) + 1, 4), (3, 5, 8, -1),
                (65535, 5, 8, 1 << 20)):
        assert L.cdsl_op_pages_workspace(*bad) == 0


def test_sizes_beyond_the_calls():
    from paper_2412_10418_amd.binding import CDSL_EINVAL, CDSL_ERANGE
    far = dict(refs=1 << 40)      # arrays of 2^30 ints that do not meet the others
    for kw in (dict(batch=65536), dict(table_stride=1 << 26), dict(pages=(1 << 30) + 1), dict(n_kv_heads=1 << 24, n_layers=1)):
        for f in CALLS:
            assert f(_cache(**kw), **far) == CDSL_ERANGE, (f.__name__, kw)
    assert _copy(_cache(n_kv_heads=1 << 24, n_layers=1)) == CDSL_ERANGE
    assert _reserve(_cache(batch=65535), table=1 << 41, refs=1 << 40, lens=1 << 42, count=1 << 43, got=1 << 44, most=1 << 20) == CDSL_ERANGE
    for kw in (dict(n_layers=3), dict(n_kv_heads=5), dict(head_dim=128), dict(format=1), dict(format=4)):
        assert _copy(_cache(), _cache(**kw)) == CDSL_EINVAL, kw


def test_empty_calls_launch_nothing():
    from paper_2412_10418_amd.binding import CDSL_OK
    none = _cache(batch=0, table=None)
    assert _fork(none, table=None, refs=None, parents=None) == CDSL_OK
    assert _reserve(none, table=None, refs=None, lens=None, count=None, got=None, ws=None, n=0) == CDSL_OK
    assert _free(none, table=None, refs=None, lens=None) == CDSL_OK
    assert _copy(_cache(), src=None, dst=None, n=0) == CDSL_OK


def test_the_plain_form_by_hand():
    """pages_ref, which the GPU tests hold the calls to, on a case that is worked out here."""
    import numpy as np

    from pages_ref import Pages
    p = Pages(np.array([[5, 2, -1], [5, 2, -1], [-1, -1, -1]]), np.array([0, 0, 2, 0, 0, 2]), np.arange(6).reshape(1, 6, 1))
    got = p.reserve([40, 40, 0], [30, 1, 100], 60)
    # page 2 is left by both: the first keeps it; its next entry is free page 0, the second's copy 1, the third prompt's 3 and 4
    assert p.table.tolist() == [[5, 2, 0], [5, 1, -1], [3, 4, -1]] and got.tolist() == [30, 1, 60]
    assert p.pool.reshape(-1).tolist() == [0, 2, 2, 3, 4, 5] and p.refs.tolist() == [1, 1, 1, 1, 1, 2]
    p.free([0, 64, 0])
    assert p.refs.tolist() == [0, 1, 0, 0, 0, 1] and p.compact() == 2
    assert p.table.tolist() == [[-1] * 3, [0, 1, -1], [-1] * 3] and p.pool.reshape(-1).tolist()[:2] == [5, 2]


def test_the_binding_checks_refs():
    from paper_2412_10418_amd import binding as bd
    with pytest.raises((ValueError, AttributeError)):
        bd.cdsl_op_pages_fork(None, torch.zeros(3, dtype=torch.int32), torch.zeros(3, dtype=torch.int32))

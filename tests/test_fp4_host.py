"""The 4-bit cache without a GPU: its layout (csrc/kvq_layout.h under AddressSanitizer and UndefinedBehaviorSanitizer), the
sizes of its pools, and its refusals, made on the host before anything is launched."""
import os
import shutil
import subprocess

import pytest
import torch

from test_tree_ops_host import P, _attend, _cache, _keep, _read, _write

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.skipif(shutil.which("g++") is None, reason="needs g++")
def test_fp4_layout_under_sanitizers(tmp_path):
    exe = tmp_path / "fp4_layout_test"
    src = os.path.join(ROOT, "tests", "native", "fp4_layout_test.cpp")
    inc = os.path.join(ROOT, "paper_2412_10418_amd", "csrc")
    cmd = ["g++", "-std=c++17", "-O1", "-g", "-fno-omit-frame-pointer", "-fsanitize=address,undefined",
           "-fno-sanitize-recover=all", "-I", inc, src, "-o", str(exe)]
    r = subprocess.run(cmd, capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=1:verify_asan_link_order=0",
               UBSAN_OPTIONS="print_stacktrace=1")
    r = subprocess.run([str(exe)], capture_output=True, text=True, env=env, timeout=120)
    assert r.returncode == 0, r.stdout + r.stderr
    assert "fp4 layout: ok" in r.stdout


def test_sizes_of_pools():
    from paper_2412_10418_amd import binding as bd
    L = bd.lib()
    for fmt, unit in ((bd.CDSL_KVQ_INT8, 64 * 128 + 256), (bd.CDSL_KVQ_E4M3, 64 * 128 + 256), (bd.CDSL_KVQ_MXFP4, 34 * 128)):
        assert L.cdsl_op_kvq_pool_bytes_of(2, 3, 4, 128, fmt) == 24 * unit
    assert L.cdsl_op_kvq_pool_bytes_of(32, 1 << 20, 8, 128, bd.CDSL_KVQ_MXFP4) == 32 * (1 << 20) * 8 * 4352
    for bad in ((0, 3, 4, 128), (2, 0, 4, 128), (2, 3, 0, 128), (2, 3, 4, 96), (-1, 3, 4, 64), (2 ** 31 - 1,) * 3 + (128,)):
        assert L.cdsl_op_kvq_pool_bytes_of(*bad, bd.CDSL_KVQ_MXFP4) == 0
    for fmt in (-1, 2, 3, 5, 2 ** 31 - 1):
        assert L.cdsl_op_kvq_pool_bytes_of(2, 3, 4, 128, fmt) == 0


@pytest.mark.parametrize("kw", [dict(pool=None), dict(table=None), dict(n_layers=0), dict(head_dim=48), dict(batch=-1), dict(pool=P + 8),
                                dict(format=3), dict(format=5)], ids=str)
def test_bad_descriptors_are_refused_by_every_call(kw):
    from paper_2412_10418_amd.binding import CDSL_EINVAL
    c = _cache(**{**dict(format=4), **kw})
    for f in (_write, _read, _attend, _keep):
        assert f(c) == CDSL_EINVAL, f.__name__


def test_sizes_at_the_ends_of_their_types():
    from paper_2412_10418_amd import binding as bd
    c = _cache(format=4, n_layers=2 ** 31 - 1, pages=2 ** 31 - 1, n_kv_heads=2 ** 31 - 1, head_dim=128)
    assert _write(c) == _read(c) == _keep(c) == _attend(c, H=2 ** 31 - 1) == bd.CDSL_ERANGE
    c = _cache(format=4, table_stride=1 << 26)
    assert _write(c) == _read(c) == _keep(c) == _attend(c) == bd.CDSL_ERANGE
    c = _cache(format=4)
    assert _write(c, T=0) == _read(c, T=0) == _attend(c, n=0) == bd.CDSL_OK
    assert _attend(c, n=513, parents=P) == bd.CDSL_ERANGE


def test_workspaces_cover_the_format():
    """The size does not ask for the format, so it has to be enough for each: a call whose keys are split refuses less."""
    from paper_2412_10418_amd import binding as bd
    for B, n, H, heads, hd, most in ((3, 1, 8, 4, 64, 30000), (1, 40, 8, 2, 128, 9000), (8, 65, 32, 8, 128, 8192)):
        need = bd.lib().cdsl_op_tree_attention_workspace(B, n, H, heads, hd, most)
        assert need > 0
        c = _cache(format=4, batch=B, n_kv_heads=heads, head_dim=hd, table_stride=1000)
        assert _attend(c, n=n, H=H, max_len=most) == bd.CDSL_EINVAL


def test_the_binding_holds_pools_to_their_format():
    from paper_2412_10418_amd import binding as bd
    table = torch.zeros((1, 2), dtype=torch.int32)
    for unit, fmt in ((64 * 64 + 256, "mxfp4"), (34 * 64, "int8"), (34 * 64, "e4m3"), (34 * 64, "mxfp4")):   # the last: on no device
        with pytest.raises(ValueError):
            bd.QuantCache(torch.zeros((1, 4, 2, unit), dtype=torch.uint8), table, 64, fmt)
    with pytest.raises(ValueError):
        bd.QuantCache.empty(1, 4, 2, 64, fmt="int4")
    with pytest.raises(ValueError):
        bd.QuantCache.empty(1, 4, 2, 96, fmt="mxfp4")
    assert bd.QuantCache.empty(1, 4, 2, 64, device="cpu", fmt="mxfp4").shape == (1, 4, 2, 34 * 64)

"""Refusals of the calls around a drafted tree (the 8-bit cache, tree
attention, verification, the kept path): every one is made on the host before
anything is launched, so they are checked here without a GPU, on pointers that
are never followed."""
import ctypes as C

import pytest
import torch

P = 0x1000      # a 16-byte aligned address that no refused call touches
OK = dict(pool=P, table=P, n_layers=2, pages=8, n_kv_heads=4, head_dim=64, batch=3, table_stride=5, format=0)


def _cache(**kw):
    from paper_2412_10418_amd.binding import KVQ
    return KVQ(**{**OK, **kw})


def _call(name, *args):
    from paper_2412_10418_amd import binding as bd
    return getattr(bd.lib(), name)(*args)


def _write(c, layer=0, K=P, V=P, dtype=0, T=4, strides=(256, 256, 256, 256), start=None, count=None):
    return _call("cdsl_op_kvq_write", C.addressof(c) if c else None, layer, K, V, dtype, T, *strides, start, count, None)


def _read(c, layer=0, K=P, V=P, dtype=0, T=4):
    return _call("cdsl_op_kvq_read", C.addressof(c) if c else None, layer, K, V, dtype, T, None, None, None)


def _attend(c, layer=0, Q=P, dtype=0, n=4, H=8, qsb=2048, qst=512, lens=P, parents=None, scale=1.0, max_len=0, out=P,
            ws=None, ws_bytes=0):
    return _call("cdsl_op_tree_attention", C.addressof(c) if c else None, layer, Q, dtype, n, H, qsb, qst, lens, None,
                 parents, scale, max_len, out, ws, ws_bytes, None)


def _accept(p=P, q=P, B=2, n=4, V=100, tokens=P, parents=P, u=P, v=P, path=P, n_path=P, token=P, ws=None,
            ws_bytes=0):
    return _call("cdsl_op_tree_accept", p, q, B, n, V, tokens, parents, None, u, v, 1, path, n_path, token, ws, ws_bytes,
                 None)


def _keep(c, lens=P, path=P, n_path=P, n=4, new=P + 64):
    return _call("cdsl_op_kvq_keep", C.addressof(c) if c else None, lens, path, n_path, n, new, None)


BAD_CACHES = [dict(pool=None), dict(table=None), dict(n_layers=0), dict(pages=0), dict(pages=-1), dict(n_kv_heads=0),
              dict(head_dim=0), dict(head_dim=48), dict(head_dim=256), dict(batch=-1), dict(table_stride=0),
              dict(format=2), dict(format=-1), dict(pool=P + 8)]


@pytest.mark.parametrize("kw", BAD_CACHES, ids=[str(k) for k in BAD_CACHES])
def test_bad_cache_descriptors_are_refused_by_every_call(kw):
    from paper_2412_10418_amd.binding import CDSL_EINVAL
    c = _cache(**kw)
    for f in (_write, _read, _attend, _keep):
        assert f(c) == CDSL_EINVAL, f.__name__


def test_null_caches_and_too_many_prompts():
    from paper_2412_10418_amd.binding import CDSL_EINVAL, CDSL_ERANGE
    for f in (_write, _read, _attend, _keep):
        assert f(None) == CDSL_EINVAL
        assert f(_cache(batch=65536)) == CDSL_ERANGE


def test_rows_that_cannot_be_written_or_read():
    from paper_2412_10418_amd.binding import CDSL_EINVAL, CDSL_ERANGE
    c = _cache()
    for f in (_write, _read):
        for kw in (dict(layer=-1), dict(layer=2), dict(K=None), dict(V=None), dict(K=P + 4), dict(V=P + 8),
                   dict(dtype=2), dict(T=-1)):
            assert f(c, **kw) == CDSL_EINVAL, (f.__name__, kw)
        assert f(_cache(n_kv_heads=32), T=2 ** 31 - 1) == CDSL_ERANGE
    for at in range(4):
        strides = [256] * 4
        strides[at] = 258                       # 1032 bytes
        assert _write(c, strides=strides) == CDSL_EINVAL
    assert _write(c, dtype=1, strides=(256, 260, 256, 256)) == CDSL_EINVAL   # 520 bytes of bf16


def test_attention_that_cannot_be_computed():
    from paper_2412_10418_amd import binding as bd
    c = _cache()
    for kw in (dict(layer=2), dict(layer=-1), dict(Q=None), dict(lens=None), dict(out=None), dict(dtype=3), dict(n=-1),
               dict(H=0), dict(H=6), dict(scale=float("nan")), dict(scale=float("inf")), dict(Q=P + 8), dict(out=P + 4),
               dict(qsb=2046), dict(qst=510), dict(dtype=1, qst=516)):
        assert _attend(c, **kw) == bd.CDSL_EINVAL, kw
    assert _attend(c, n=513, parents=P) == bd.CDSL_ERANGE
    assert _attend(c, n=2 ** 28, H=8) == bd.CDSL_ERANGE
    assert _attend(c, n=2 ** 21, H=8) == bd.CDSL_ERANGE        # 3 prompts of 2^24 rows
    # a call that splits its keys needs its workspace
    need = bd.lib().cdsl_op_tree_attention_workspace(3, 1, 8, 4, 64, 30000)
    assert need > 0
    for ws, size in ((None, 0), (P, need - 1), (None, need)):
        assert _attend(c, n=1, max_len=30000, ws=ws, ws_bytes=size) == bd.CDSL_EINVAL
    assert _attend(c, n=1, max_len=30000, ws=P + 4, ws_bytes=need) == bd.CDSL_EINVAL


def test_trees_that_cannot_be_verified():
    from paper_2412_10418_amd.binding import CDSL_EINVAL, CDSL_ERANGE
    for kw in (dict(p=None), dict(q=None), dict(tokens=None), dict(parents=None), dict(u=None), dict(v=None),
               dict(path=None), dict(n_path=None), dict(token=None), dict(B=-1), dict(n=0), dict(V=0)):
        assert _accept(**kw) == CDSL_EINVAL, kw
    assert _accept(n=513) == CDSL_ERANGE
    assert _accept(V=(1 << 20) + 1) == CDSL_ERANGE
    assert _accept(B=65536) == CDSL_ERANGE
    # long rows need their workspace
    from paper_2412_10418_amd import binding as bd
    need = bd.lib().cdsl_op_tree_accept_workspace(2, 4, 128256)
    assert need > 0 and bd.lib().cdsl_op_tree_accept_workspace(2, 4, 32000) == 0
    for ws, size in ((None, 0), (P, need - 1), (None, need), (P + 8, need)):
        assert _accept(V=128256, ws=ws, ws_bytes=size) == CDSL_EINVAL
    for bad in ((0, 4, 128256), (2, 0, 128256), (2, 513, 128256), (2, 4, 0), (2, 4, (1 << 20) + 1)):
        assert bd.lib().cdsl_op_tree_accept_workspace(*bad) == 0


def test_paths_that_cannot_be_kept():
    from paper_2412_10418_amd.binding import CDSL_EINVAL, CDSL_ERANGE
    c = _cache()
    for kw in (dict(lens=None), dict(path=None), dict(n_path=None), dict(n=-1), dict(new=P)):
        assert _keep(c, **kw) == CDSL_EINVAL, kw
    assert _keep(_cache(n_layers=1 << 20, n_kv_heads=1 << 10)) == CDSL_ERANGE


def test_empty_calls_launch_nothing():
    from paper_2412_10418_amd.binding import CDSL_OK
    none = _cache(batch=0, table=None)
    assert _write(none, K=None, V=None) == CDSL_OK and _write(_cache(), K=None, V=None, T=0) == CDSL_OK
    assert _read(none, K=None, V=None) == CDSL_OK and _read(_cache(), T=0) == CDSL_OK
    assert _attend(none, Q=None, lens=None, out=None) == CDSL_OK and _attend(_cache(), n=0) == CDSL_OK
    assert _accept(B=0, p=None, q=None) == CDSL_OK
    assert _keep(none, lens=None, path=None, n_path=None, new=None) == CDSL_OK


def test_sizes():
    from paper_2412_10418_amd import binding as bd
    L = bd.lib()
    assert L.cdsl_op_kvq_pool_bytes(2, 3, 4, 128) == 24 * (64 * 128 + 256)
    assert L.cdsl_op_kvq_pool_bytes(32, 1 << 20, 8, 128) == 32 * (1 << 20) * 8 * 8448     # beyond 2^32
    for bad in ((0, 3, 4, 128), (2, 0, 4, 128), (2, 3, 0, 128), (2, 3, 4, 96), (-1, 3, 4, 64)):
        assert L.cdsl_op_kvq_pool_bytes(*bad) == 0
    for bad in ((0, 1, 8, 8, 64, 9), (1, 0, 8, 8, 64, 9), (1, 1, 7, 2, 64, 9), (1, 1, 0, 1, 64, 9), (1, 1, 8, 0, 64, 9)):
        assert L.cdsl_op_tree_attention_workspace(*bad) == 0
    # short contexts, and batches that fill the chip, are not split
    assert L.cdsl_op_tree_attention_workspace(1, 1, 32, 8, 64, 64) == 0
    assert L.cdsl_op_tree_attention_workspace(64, 65, 32, 8, 128, 2048) == 0
    # a bound below 0 counts as none
    assert L.cdsl_op_tree_attention_workspace(1, 1, 32, 8, 64, -5) == L.cdsl_op_tree_attention_workspace(1, 1, 32, 8, 64, 0)


def test_the_binding_refuses_what_the_library_cannot_see():
    from paper_2412_10418_amd import binding as bd
    pool, table = torch.zeros((1, 4, 2, 64 * 64 + 256), dtype=torch.uint8), torch.zeros((1, 2), dtype=torch.int32)
    for args in ((pool, table, 64, "int8"),              # not on a device
                 (pool, table, 64, "int4"), (pool, table, 48, "int8"), (pool[0], table, 64, "int8"),
                 (pool, table[0], 64, "int8")):
        with pytest.raises(ValueError):
            bd.QuantCache(*args)
    with pytest.raises(ValueError):
        bd.QuantCache.empty(1, 4, 2, 96)
    with pytest.raises(ValueError):
        bd.cdsl_op_tree_accept(torch.zeros(1, 2, 3), torch.zeros(1, 2, 3), table, table, torch.zeros(1, 2), torch.zeros(1))

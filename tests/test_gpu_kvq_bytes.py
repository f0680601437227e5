"""The 8-bit cache byte by byte: what writes and kept paths leave in the whole pool (pages and slots that no prompt has
among it), against the layout's formulas on the host."""
import numpy as np
import pytest
import torch

from test_gpu_tree_ops import FMTS, _ints, _np, _rows
from tree_ref import TINY, paged

pytestmark = pytest.mark.gpu


def _places(hd):
    """[32, 2 hd + 8]: where in a unit the bytes of a slot's key, value, key scale and value scale stand."""
    s, d, b = np.arange(32)[:, None], np.arange(hd)[None, :], np.arange(4)[None, :]
    key = d // 32 * 1024 + d % 32 // 8 * 256 + s % 16 * 16 + s // 16 * 8 + d % 8
    value = 32 * hd + d // 32 * 1024 + s % 16 // 4 * 256 + d % 16 * 16 + d % 32 // 16 * 8 + s // 16 * 4 + s % 4
    return np.concatenate([key, value, 64 * hd + 4 * s + b, 64 * hd + 128 + 4 * s + b], 1)


def _scales(x, fmt):
    a = np.abs(x.astype(np.float64)).max(-1)
    if fmt == "int8":
        return np.maximum((a / 127).astype(np.float32), np.float32(TINY))
    with np.errstate(divide="ignore"):
        e = np.where(a > 0, np.ceil(np.log2(a / 448)), -200)
    return np.maximum(2.0 ** np.maximum(e, -126), TINY).astype(np.float32)


def _bytes(x, fmt):
    """Codes [..., hd] (bytes) and scales [..., 4] of rows x (numpy, fp32)."""
    s = _scales(x, fmt)
    y = x.astype(np.float64) / s[..., None].astype(np.float64)
    if fmt == "int8":
        code = np.rint(y).astype(np.int8).view(np.uint8)
    else:   # quotients by a power of two are exact in fp32
        code = torch.from_numpy(y.astype(np.float32)).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    return code, s[..., None].view(np.uint8)


def _slots(table, b, positions):
    return table[b, positions // 32], positions % 32


def _row_bytes(pool, layer, page, slot, places):
    return pool[layer, page][:, places[slot]]             # [heads, 2 hd + 8]


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("B,T,heads,hd,start", [(1, 1, 8, 128, 95), (3, 33, 2, 64, 31), (2, 64, 5, 128, 32), (4, 70, 3, 32, 7),
                                                (2, 130, 1, 64, 0)])
def test_writes_change_the_bytes_of_their_rows_alone(fmt, kind, B, T, heads, hd, start):
    from paper_2412_10418_amd import binding as bd
    rng = np.random.default_rng([T, heads, hd, start])
    cache = paged(rng, 2, B, start + T + 9, heads, hd, fmt, spare=3)
    K, V = _rows(rng, (B, T, heads, hd), kind), _rows(rng, (B, T, heads, hd), kind)
    at, count = start + rng.integers(0, 9, B), rng.integers(0, T + 1, B)
    count[0] = T
    want, table, places = cache.pool.cpu().numpy(), cache.table.cpu().numpy(), _places(hd)
    bd.cdsl_op_kvq_write(cache, K, V, start=_ints(at), count=_ints(count), layer=1)
    (kc, ks), (vc, vs) = _bytes(_np(K), fmt), _bytes(_np(V), fmt)
    rows = np.concatenate([kc, vc, ks, vs], -1)           # [B, T, heads, 2 hd + 8]
    for b in range(B):
        for t in range(count[b]):
            page, slot = _slots(table, b, at[b] + t)
            want[1, page][:, places[slot]] = rows[b, t]
    assert np.array_equal(cache.pool.cpu().numpy(), want)


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("B,n,heads,hd,layers", [(1, 1, 1, 32, 1), (3, 12, 2, 64, 2), (2, 70, 5, 128, 3), (4, 200, 1, 32, 2),
                                                 (5, 33, 2, 128, 2)])
def test_kept_paths_change_the_bytes_of_their_slots_alone(fmt, B, n, heads, hd, layers):
    """The pool holds arbitrary bytes: moves are of bytes, whatever they mean."""
    from paper_2412_10418_amd import binding as bd
    rng = np.random.default_rng([n, hd, 7])
    lens = rng.integers(0, 70, B)
    cache = paged(rng, layers, B, 70 + n, heads, hd, fmt, spare=3)
    m = rng.integers(1, n + 1, B)
    path = np.full((B, n), -1, np.int32)
    for b in range(B):
        path[b, :m[b]] = np.sort(rng.permutation(n)[:m[b]])
    old, table, places = cache.pool.cpu().numpy(), cache.table.cpu().numpy(), _places(hd)
    want = old.copy()
    bd.cdsl_op_kvq_keep(cache, _ints(lens), _ints(path), _ints(m))
    for layer in range(layers):
        for b in range(B):
            for i in range(m[b]):
                page, slot = _slots(table, b, lens[b] + path[b, i])
                to, at = _slots(table, b, lens[b] + i)
                want[layer, to][:, places[at]] = _row_bytes(old, layer, page, slot, places)
    assert np.array_equal(cache.pool.cpu().numpy(), want)

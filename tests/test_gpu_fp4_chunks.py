"""Chunks of a prompt over the 4-bit cache, long enough that rows see whole pages of the chunk itself: against the 64-bit form,
and with rows of the chunk that are NaN."""
import numpy as np
import pytest
import torch

from fp4_ref import paged
from test_gpu_tree_ops import KIND, _check, _ints, _np, _rows

pytestmark = pytest.mark.gpu

CASES = [  # B, n, H, heads, hd, lens: tiles of 16 rows; the same at odd group sizes; two waves a tile, 57 row groups a pair
    (1, 300, 4, 1, 128, [77]), (2, 130, 6, 2, 64, [40, 0]), (1, 900, 32, 8, 32, [200]), (1, 900, 32, 8, 128, [157]),
]
IDS = [f"{c[0]}x{c[1]}-{c[2]}.{c[3]}x{c[4]}" for c in CASES]


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("case", CASES, ids=IDS)
def test_chunks_match_their_definition(case, kind):
    from paper_2412_10418_amd import binding as bd
    B, n, H, heads, hd, lens = case
    rng = np.random.default_rng([n, H, hd, 77])
    T = max(lens) + n
    cache = paged(rng, 1, B, T, heads, hd)
    nodes = [n] + [n - 31] * (B - 1)
    count = _ints([l + m for l, m in zip(lens, nodes)])
    bd.cdsl_op_kvq_write(cache, *(_rows(rng, (B, T, heads, hd), kind) for _ in range(2)), count=count)
    k, v = (_np(x).astype(np.float64) for x in bd.cdsl_op_kvq_read(cache, T, count=count))
    q = (1.5 * _rows(rng, (B, n, H, hd), "f32")).to(KIND[kind])
    out = torch.full_like(q, 7.0)
    bd.cdsl_op_tree_attention(cache, q, _ints(lens), n_nodes=_ints(nodes), max_len=max(lens), out=out)
    _check(out, q, k, v, lens, None, nodes, hd ** -0.5, f"chunk {kind}")
    for b in range(B):
        assert bool((out[b, nodes[b]:] == 7).all())


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("which", ["key", "value"])
@pytest.mark.parametrize("at", [0, 41, 126])
@pytest.mark.parametrize("case", CASES, ids=IDS)
def test_a_row_of_the_chunk_that_is_nan(case, at, which, kind):
    """The rows before it are what they are without it, to the bit; it and those behind it are NaN.  With a page of the chunk
    outside the pool, the rows from that page's first on are NaN."""
    from paper_2412_10418_amd import binding as bd
    B, n, H, heads, hd, lens = case
    rng = np.random.default_rng([n, H, hd, 78])
    T = max(lens) + n
    cache = paged(rng, 1, B, T, heads, hd)
    K, V = (_rows(rng, (B, T, heads, hd), kind) for _ in range(2))
    q = _rows(rng, (B, n, H, hd), "f32").to(KIND[kind])
    outs = []
    for bad in (False, True):
        if bad:
            (K if which == "key" else V)[0, lens[0] + at, :, hd // 2 + 1] = float("nan")
        bd.cdsl_op_kvq_write(cache, K, V)
        outs.append(bd.cdsl_op_tree_attention(cache, q, _ints(lens), max_len=max(lens)))
    assert torch.isfinite(outs[0]).all()
    assert torch.equal(outs[0][0, :at], outs[1][0, :at]) and torch.equal(outs[0][1:], outs[1][1:])
    assert torch.isnan(outs[1][0, at:]).all()
    page = (lens[0] + at) // 32
    cache.table[0, page] = cache.pool.shape[1]
    gone = bd.cdsl_op_tree_attention(cache, q, _ints(lens), max_len=max(lens))
    first = max(page * 32 - lens[0], 0)
    assert torch.equal(outs[0][0, :first], gone[0, :first]) and torch.isnan(gone[0, first:]).all()

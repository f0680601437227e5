"""Every kernel of the attention over the 4-bit cache (the shapes of fp4_cases.py, whose plan test_fp4_plan_host.py checks),
entry by entry against the 64-bit form: trees and chunks, prompts with fewer nodes, rows behind them."""
import numpy as np
import pytest
import torch

from fp4_cases import params
from fp4_ref import paged
from test_gpu_tree_ops import KIND, _check, _ints, _np, _rows
from tree_ref import random_tree

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("causal", [False, True], ids=["tree", "causal"])
@pytest.mark.parametrize("case,kind", params())
def test_kernels_entry_by_entry(case, kind, causal):
    from paper_2412_10418_amd import binding as bd
    rng = np.random.default_rng([case.B, case.n, case.H, 74])
    B, n, lens = case.B, case.n, case.lens(rng)
    T = max(lens) + n
    cache = paged(rng, 1, B, T, case.heads, case.hd)
    K, V = (_rows(rng, (B, T, case.heads, case.hd), kind) for _ in range(2))
    nodes = rng.integers(0, n + 1, B)
    nodes[0], nodes[-1] = n, max(1, n - 1)
    count = _ints([l + int(m) for l, m in zip(lens, nodes)])
    bd.cdsl_op_kvq_write(cache, K, V, count=count)
    k, v = bd.cdsl_op_kvq_read(cache, T, count=count)
    q = (1.5 * _rows(rng, (B, n, case.H, case.hd), "f32")).to(KIND[kind])
    parents = None if causal else np.stack([random_tree(rng, n, 3) for _ in range(B)])
    out = torch.full_like(q, 7.0)
    bd.cdsl_op_tree_attention(cache, q, _ints(lens), None if causal else _ints(parents), n_nodes=_ints(nodes),
                              max_len=case.longest, out=out)
    some = sorted({0, B - 1})
    _check(out[some], q[some], _np(k[some]).astype(np.float64), _np(v[some]).astype(np.float64), [lens[b] for b in some],
           None if causal else parents[some], nodes[some].tolist(), case.hd ** -0.5, f"{case.name} {kind}")
    for b in range(B):
        assert torch.isfinite(out[b, :nodes[b]]).all() and bool((out[b, nodes[b]:] == 7).all())


@pytest.mark.parametrize("case,kind", params())
def test_what_is_not_seen_may_hold_anything(case, kind):
    """A pool of bytes 255 (NaN scales) around the written rows, and a NaN row in the last node of the first prompt (key) and of
    the last one (value): a star's other nodes do not see it, and stay what they are without it, to the bit."""
    from paper_2412_10418_amd import binding as bd
    rng = np.random.default_rng([case.B, case.n, case.H, 75])
    B, n, lens = case.B, case.n, case.lens(rng)
    T = max(lens) + n
    K, V = (_rows(rng, (B, T, case.heads, case.hd), kind) for _ in range(2))
    q = _rows(rng, (B, n, case.H, case.hd), "f32").to(KIND[kind])
    parents = _ints(np.tile([-1] + [0] * (n - 1), (B, 1)))
    count = _ints([l + n for l in lens])
    outs = []
    for bad in (False, True):
        cache = paged(np.random.default_rng(1), 1, B, T, case.heads, case.hd, fill=255)
        if bad:
            K[0, lens[0] + n - 1, :, 3] = float("nan")
            V[-1, lens[-1] + n - 1, :, case.hd - 1] = float("inf")
        bd.cdsl_op_kvq_write(cache, K, V, count=count)
        outs.append(bd.cdsl_op_tree_attention(cache, q, _ints(lens), parents, max_len=case.longest))
    assert torch.isfinite(outs[0]).all()
    assert torch.isnan(outs[1][0, n - 1]).all() and torch.isnan(outs[1][-1, n - 1]).all()
    if n > 1:
        assert torch.equal(outs[0][0, :n - 1], outs[1][0, :n - 1]) and torch.equal(outs[0][-1, :n - 1], outs[1][-1, :n - 1])
    assert torch.equal(outs[0][1:-1], outs[1][1:-1])


@pytest.mark.parametrize("case,kind", params())
def test_pages_that_do_not_exist_are_nan_where_they_are_seen(case, kind):
    """A page of the first prompt's tokens is missing: all its rows are NaN, the other prompts' the same to the bit."""
    from paper_2412_10418_amd import binding as bd
    rng = np.random.default_rng([case.B, case.n, case.H, 76])
    B, n, lens = case.B, case.n, case.lens(rng)
    T = max(lens) + n
    cache = paged(rng, 1, B, T, case.heads, case.hd)
    K, V = (_rows(rng, (B, T, case.heads, case.hd), kind) for _ in range(2))
    bd.cdsl_op_kvq_write(cache, K, V)
    q = _rows(rng, (B, n, case.H, case.hd), "f32").to(KIND[kind])
    good = bd.cdsl_op_tree_attention(cache, q, _ints(lens), max_len=case.longest)
    cache.table[0, 0] = cache.pool.shape[1]
    got = bd.cdsl_op_tree_attention(cache, q, _ints(lens), max_len=case.longest)
    assert torch.isnan(got[0]).all() and torch.equal(got[1:], good[1:])

"""Every kernel of the tree attention at heads of 128 (the shapes of tree_cases.py, whose plan test_tree_plan_host.py
checks), entry by entry against the 64-bit form: trees and chunks, prompts with fewer nodes, rows behind them."""
import numpy as np
import pytest
import torch

from test_gpu_tree_ops import KIND, _check, _ints, _np, _rows
from tree_cases import params
from tree_ref import paged, random_tree

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("causal", [False, True], ids=["tree", "causal"])
@pytest.mark.parametrize("case,kind,fmt", params())
def test_kernels_entry_by_entry(case, kind, fmt, causal):
    from paper_2412_10418_amd import binding as bd
    rng = np.random.default_rng([case.B, case.n, case.H, 73])
    B, n, lens = case.B, case.n, case.lens(rng)
    T = max(lens) + n
    cache = paged(rng, 1, B, T, case.heads, case.hd, fmt)
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
           None if causal else parents[some], nodes[some].tolist(), case.hd ** -0.5, f"{case.name} {kind} {fmt}")
    for b in range(B):
        assert torch.isfinite(out[b, :nodes[b]]).all() and bool((out[b, nodes[b]:] == 7).all())

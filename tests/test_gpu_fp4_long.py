"""Prompts whose pages outnumber the ids that a wave holds at a time, unsplit, among prompts of one token: the long ones entry by
entry against the 64-bit form (fp4_cases.MANY_PAGES, whose kernels test_fp4_plan_host.py checks)."""
import numpy as np
import pytest
import torch

from fp4_cases import KINDS, MANY_PAGES
from test_gpu_tree_ops import KIND, _check, _ints, _np, _rows

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("case", MANY_PAGES, ids=[c.name.replace(" ", "_") for c in MANY_PAGES])
def test_prompts_of_many_pages(case, kind):
    from paper_2412_10418_amd import binding as bd
    rng = np.random.default_rng([case.B, case.n, case.hd, 76])
    B, n, heads, hd = case.B, case.n, case.heads, case.hd
    long = {0: case.longest, B - 1: case.longest - 37}
    lens = [long.get(b, 1) for b in range(B)]
    per = [-(-(L + n) // 32) for L in lens]
    P = max(per)
    ids = rng.permutation(sum(per))
    table = np.full((B, P), -1, np.int32)
    for b, at in enumerate(np.cumsum([0] + per[:-1])):
        table[b, :per[b]] = ids[at:at + per[b]]
    table = _ints(table)
    pool = bd.QuantCache.empty(1, len(ids), heads, hd, fmt="mxfp4")
    k, v = {}, {}
    for b in range(B):
        one = bd.QuantCache(pool, table[b:b + 1], hd, "mxfp4")
        T = lens[b] + n
        bd.cdsl_op_kvq_write(one, *(_rows(rng, (1, T, heads, hd), kind) for _ in range(2)))
        if b in long:
            k[b], v[b] = (_np(x[0]).astype(np.float64) for x in bd.cdsl_op_kvq_read(one, T))
    q = (1.5 * _rows(rng, (B, n, case.H, hd), "f32")).to(KIND[kind])
    out = bd.cdsl_op_tree_attention(bd.QuantCache(pool, table, hd, "mxfp4"), q, _ints(lens), max_len=case.longest)
    assert torch.isfinite(out).all()
    some = sorted(long)
    _check(out[some], q[some], [k[b] for b in some], [v[b] for b in some], [lens[b] for b in some], None, [n] * 2,
           hd ** -0.5, f"{case.name} {kind}")

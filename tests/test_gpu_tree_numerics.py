"""What the tree attention and the verification hold of their numbers, against 64-bit forms."""
import numpy as np
import pytest
import torch

from test_gpu_tree_ops import KIND, _check, _ints, _np, _rows
from tree_cases import WHOLE, params
from tree_ref import paged, random_tree

pytestmark = pytest.mark.gpu


def _filled(rng, case, fmt):
    """The case's cache, the prompt lengths, and the keys and values of its first and last prompt in float64."""
    from paper_2412_10418_amd import binding as bd
    lens = case.lens(rng)
    T = max(lens) + case.n
    cache = paged(rng, 1, case.B, T, case.heads, case.hd, fmt)
    K, V = (_rows(rng, (case.B, T, case.heads, case.hd), "f32") for _ in range(2))
    count = _ints([l + case.n for l in lens])
    bd.cdsl_op_kvq_write(cache, K, V, count=count)
    k, v = bd.cdsl_op_kvq_read(cache, T, count=count)
    some = sorted({0, case.B - 1})
    return cache, lens, some, _np(k[some]).astype(np.float64), _np(v[some]).astype(np.float64)


@pytest.mark.parametrize("scale", [1e-8, -1e-30, 1e30, 3e38])
@pytest.mark.parametrize("case,kind,fmt", params(WHOLE))
def test_queries_and_scales_of_any_size(case, kind, fmt, scale):
    """A row of zeros and, under the small scales, rows of 1e-20 and of 1e-40 (their scores are 0 in effect: the mean of
    what is visible) on pages that hold hidden slots, beside ordinary rows."""
    from paper_2412_10418_amd import binding as bd
    rng = np.random.default_rng([case.B, case.n, 71])
    cache, lens, some, k, v = _filled(rng, case, fmt)
    q = _rows(rng, (case.B, case.n, case.H, case.hd), "f32")
    q[:, 0] = 0
    if scale < 1:
        q[:, -1, ::2] *= 1e-20
        q[:, -1, 1::2] *= 1e-40
    else:
        q[:] = 0
    q = q.to(KIND[kind])
    parents = np.stack([random_tree(rng, case.n, 3) for _ in range(case.B)])
    out = bd.cdsl_op_tree_attention(cache, q, _ints(lens), _ints(parents), scale=scale, max_len=case.longest)
    _check(out[some], q[some], k, v, [lens[b] for b in some], parents[some], [case.n] * len(some), scale,
           f"{case.name} {kind} {fmt} {scale}")
    assert torch.isfinite(out).all()

"""Tree attention with softmax scales at the ends of fp32 and queries and keys that bring their scores to ordinary size, against
the 64-bit form (tree_ref.attention, bounds: tree_ref.tolerance)."""
import numpy as np
import pytest
import torch

from test_gpu_tree_ops import KIND, _check, _ints, _np, _rows
from tree_cases import WHOLE, params
from tree_ref import paged, random_tree

pytestmark = pytest.mark.gpu

# The powers of two of q and of the keys, and the scale: subnormal, with three and six bits left when it is multiplied by
# log2(e) in fp32; near the largest number, which that product passes.
SIZES = [(80, 66, 2.0 ** -147), (70, 70, -2.0 ** -143), (-70, -60, 3.3e38), (-50, -81, -2.5e38)]


@pytest.mark.parametrize("case,kind,fmt", params([c for c in WHOLE if "chip" not in c.name]))
def test_scales_at_the_ends_of_fp32(case, kind, fmt):
    from paper_2412_10418_amd import binding as bd
    rng = np.random.default_rng([case.B, case.n, case.hd, 83])
    lens = case.lens(rng)
    T = max(lens) + case.n
    cache = paged(rng, 1, case.B, T, case.heads, case.hd, fmt)
    K, V = (_rows(rng, (case.B, T, case.heads, case.hd), "f32") for _ in range(2))
    count = _ints([l + case.n for l in lens])
    some = sorted({0, case.B - 1})
    parents = np.stack([random_tree(rng, case.n, 3) for _ in range(case.B)])
    q = _rows(rng, (case.B, case.n, case.H, case.hd), "f32")
    for of_q, of_k, scale in SIZES:
        bd.cdsl_op_kvq_write(cache, K * 2.0 ** of_k, V, count=count)
        k, v = (_np(x[some]).astype(np.float64) for x in bd.cdsl_op_kvq_read(cache, T, count=count))
        x = (q * 2.0 ** of_q).to(KIND[kind])
        out = bd.cdsl_op_tree_attention(cache, x, _ints(lens), _ints(parents), scale=scale, max_len=case.longest)
        _check(out[some], x[some], k, v, [lens[b] for b in some], parents[some], [case.n] * len(some), scale,
               f"{case.name} {kind} {fmt} {scale}")
        assert torch.isfinite(out).all()

"""What the attention over the 4-bit cache holds of its numbers, against the 64-bit form, in the mean square: a bound entry by
entry (tree_ref.tolerance) has room for a plane of q or of the probabilities that is lost."""
import numpy as np
import pytest
import torch

from fp4_cases import params
from fp4_ref import paged
from test_gpu_tree_ops import KIND, _ints, _np, _rows
from tree_cases import rms
from tree_ref import attention, random_tree

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("case,kind", params())
def test_results_are_as_near_as_their_products(case, kind):
    """Queries of full significands; then with an entry in every row, in a channel in which the keys are 0, of 1e5 (bf16: 2^20)
    times the others' size: no other entry may lose by it.

    fp32: a score (size s, 1.4 here) is a sum of 3 hd products of planes, each addition off by at most 2^-24 s and by 0.3 of
    that in the mean square: at heads of 128 20 x 0.3 x 1.4 x 2^-24 = 5e-7 of a probability; its exponential and the sums over
    the keys as much again: 1e-6 in all.  (Two planes of q or of the probabilities would give 3e-6 and more:
    test_fp4_numerics_host.py.)  bf16: beside the results' own rounding each probability is rounded, by itself and by half a
    step, 2^-8 of it, at most, so in a sum of independent terms the mean square grows by 2^-16 of the results' at most.  With 16
    rows a KV head or fewer it is off by 2^-16 at most, and so is the result but for its own rounding (1% of which is for the
    roundings that fall to the other side)."""
    from paper_2412_10418_amd import binding as bd
    rng = np.random.default_rng([case.B, case.n, case.hd, 72])
    lens = case.lens(rng)
    T = max(lens) + case.n
    cache = paged(rng, 1, case.B, T, case.heads, case.hd)
    K, V = (_rows(rng, (case.B, T, case.heads, case.hd), "f32") for _ in range(2))
    K[..., 5] = 0
    count = _ints([l + case.n for l in lens])
    bd.cdsl_op_kvq_write(cache, K, V, count=count)
    some = sorted({0, case.B - 1})
    k, v = (_np(x[some]).astype(np.float64) for x in bd.cdsl_op_kvq_read(cache, T, count=count))
    parents = np.stack([random_tree(rng, case.n, 3) for _ in range(case.B)])
    q = 0.5 * torch.from_numpy(rng.standard_normal((case.B, case.n, case.H, case.hd), np.float32)).cuda()
    for outlier in (0, 1e5 if kind == "f32" else 2.0 ** 20):
        if outlier:
            q[..., 5] = outlier * torch.from_numpy(rng.choice(np.float32([-1.7, -1, 1, 1.3]), q.shape[:3])).cuda()
        x = q.to(KIND[kind])
        out = _np(bd.cdsl_op_tree_attention(cache, x, _ints(lens), _ints(parents), max_len=case.longest))
        off, own, ref = [], [], []
        for i, b in enumerate(some):
            o, _, _ = attention(_np(x[b]).astype(np.float64), k[i][:lens[b] + case.n], v[i][:lens[b] + case.n], lens[b],
                                parents[b], case.hd ** -0.5)
            off.append((out[b] - o).ravel())
            own.append((_np(torch.from_numpy(o).to(KIND[kind])) - o).ravel())
            ref.append(o.ravel())
        off, own, ref = (rms(np.concatenate(y)) for y in (off, own, ref))
        print(f"{case.name} {kind} {outlier}: off by {off / ref:.3g} of the results, their own rounding {own / ref:.3g}", flush=True)
        if kind == "f32":
            assert off <= 1e-6 * ref
        elif case.kernel(kind, "mxfp4").startswith("few1"):
            assert off <= 1.01 * own + 2.0 ** -16 * ref
        else:
            assert off ** 2 <= own ** 2 + (2.0 ** -8 * ref) ** 2

"""Attention over the 4-bit cache with queries, keys and softmax scales of any size, against the 64-bit form (tree_ref.attention,
bounds: tree_ref.tolerance)."""
import numpy as np
import pytest
import torch

from fp4_cases import ALL
from fp4_ref import paged
from test_gpu_tree_ops import KIND, _check, _ints, _np, _rows
from tree_cases import KINDS
from tree_ref import random_tree

pytestmark = pytest.mark.gpu


def params(names):
    return [pytest.param(c, k, id=f"{c.name}-{k}".replace(" ", "_")) for c in ALL if c.name in names for k in KINDS]


def _filled(rng, case, size=0):
    """The case's cache with keys around 2^size, the prompt lengths, and what its first and last prompt read back, in float64."""
    from paper_2412_10418_amd import binding as bd
    lens = case.lens(rng)
    T = max(lens) + case.n
    cache = paged(rng, 1, case.B, T, case.heads, case.hd)
    K, V = (_rows(rng, (case.B, T, case.heads, case.hd), "f32") for _ in range(2))
    count = _ints([l + case.n for l in lens])
    bd.cdsl_op_kvq_write(cache, K * 2.0 ** size, V, count=count)
    k, v = bd.cdsl_op_kvq_read(cache, T, count=count)
    some = sorted({0, case.B - 1})
    return cache, lens, some, _np(k[some]).astype(np.float64), _np(v[some]).astype(np.float64)


# The powers of two of q, of the keys and of the scale, q . k in fp32's range; scores are ordinary, or so small that all weights
# are alike (scales that are subnormal, to the smallest).
SIZES = [(36, 82, -140), (100, 18, -149), (90, 28, -128), (112, -106, -9)]
KERNELS = ("few1", "few1 hd32", "few2", "few2 hd64", "many", "many hd32", "wide", "wide hd64", "paired", "paired hd32",
           "few1 split", "wide split hd32")


@pytest.mark.parametrize("case,kind", params(KERNELS))
def test_scores_of_ordinary_size_whatever_their_factors(case, kind):
    from paper_2412_10418_amd import binding as bd
    for i, (of_q, of_k, of_scale) in enumerate(SIZES):
        rng = np.random.default_rng([case.B, case.n, case.hd, 81])
        cache, lens, some, k, v = _filled(rng, case, of_k)
        q = (_rows(rng, (case.B, case.n, case.H, case.hd), "f32") * 2.0 ** of_q).to(KIND[kind])
        scale = (-1) ** i * 2.0 ** of_scale
        parents = np.stack([random_tree(rng, case.n, 3) for _ in range(case.B)])
        out = bd.cdsl_op_tree_attention(cache, q, _ints(lens), _ints(parents), scale=scale, max_len=case.longest)
        _check(out[some], q[some], k, v, [lens[b] for b in some], parents[some], [case.n] * len(some), scale,
               f"{case.name} {kind} {SIZES[i]}")
        assert torch.isfinite(out).all()


# q . k beyond fp32 or below its normal numbers; subnormal q.
BEYOND = [(20, 110, 2.0 ** -133), (70, 70, -2.0 ** -143), (-70, -60, 3.3e38), (-64, -60, -2.0 ** 121), (-135, 10, 2.0 ** 122)]


@pytest.mark.parametrize("case,kind", params(KERNELS))
def test_scores_of_ordinary_size_by_way_of_sums_beyond_fp32(case, kind):
    """Rows of q are as if scaled to entries below 2; what they are times keys below 2^119 is in range."""
    from paper_2412_10418_amd import binding as bd
    for of_q, of_k, scale in BEYOND:
        rng = np.random.default_rng([case.B, case.n, case.hd, 84])
        cache, lens, some, k, v = _filled(rng, case, of_k)
        q = (_rows(rng, (case.B, case.n, case.H, case.hd), "f32") * 2.0 ** of_q).to(KIND[kind])
        parents = np.stack([random_tree(rng, case.n, 3) for _ in range(case.B)])
        out = bd.cdsl_op_tree_attention(cache, q, _ints(lens), _ints(parents), scale=scale, max_len=case.longest)
        _check(out[some], q[some], k, v, [lens[b] for b in some], parents[some], [case.n] * len(some), scale,
               f"{case.name} {kind} {of_q} {of_k} {scale}")
        assert torch.isfinite(out).all()


@pytest.mark.parametrize("case,kind", params(("few1", "few2", "many", "wide", "paired hd32")))
def test_scaling_a_row_by_powers_of_two_changes_no_bit(case, kind):
    """q times 2^a under a scale times 2^-a: what is taken of the entries does not depend on their row's size."""
    from paper_2412_10418_amd import binding as bd
    rng = np.random.default_rng([case.B, case.n, case.hd, 85])
    cache, lens, _, _, _ = _filled(rng, case)
    q = _rows(rng, (case.B, case.n, case.H, case.hd), "f32").to(KIND[kind])
    ref = bd.cdsl_op_tree_attention(cache, q, _ints(lens), scale=0.125, max_len=case.longest)
    for a in (-90, -1, 1, 30, 110):
        got = bd.cdsl_op_tree_attention(cache, q * 2.0 ** a, _ints(lens), scale=0.125 * 2.0 ** -a, max_len=case.longest)
        assert torch.equal(got, ref), a


@pytest.mark.parametrize("scale", [0.0, 1e-8, -1e-30, 1e30, 3e38])
@pytest.mark.parametrize("case,kind", params(("few1", "few2", "many", "wide", "paired hd32")))
def test_queries_and_scales_of_any_size(case, kind, scale):
    """A row of zeros and, under the small scales, rows of 1e-20 and of 1e-40 (their scores are 0 in effect: the mean of
    what is visible) on pages that hold hidden slots, beside ordinary rows."""
    from paper_2412_10418_amd import binding as bd
    rng = np.random.default_rng([case.B, case.n, case.hd, 82])
    cache, lens, some, k, v = _filled(rng, case)
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
           f"{case.name} {kind} {scale}")
    assert torch.isfinite(out).all()

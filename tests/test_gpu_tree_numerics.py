"""What the tree attention and the verification hold of their numbers, against 64-bit forms."""
import numpy as np
import pytest
import torch

from test_gpu_tree_ops import KIND, _check, _ints, _np, _rows, _verify
from tree_cases import ALL, WHOLE, params, rms
from tree_ref import attention, paged, random_tree

pytestmark = pytest.mark.gpu


def _filled(rng, case, fmt, quiet=None):
    """The case's cache, the prompt lengths, and the keys and values of its first and last prompt in float64.  quiet: a
    channel in which all keys are 0."""
    from paper_2412_10418_amd import binding as bd
    lens = case.lens(rng)
    T = max(lens) + case.n
    cache = paged(rng, 1, case.B, T, case.heads, case.hd, fmt)
    K, V = (_rows(rng, (case.B, T, case.heads, case.hd), "f32") for _ in range(2))
    if quiet is not None:
        K[..., quiet] = 0
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


@pytest.mark.parametrize("outlier", [0, 1e3, 1e5])
@pytest.mark.parametrize("case,kind,fmt", params(ALL))
def test_results_are_as_near_as_their_products(case, kind, fmt, outlier):
    """With `outlier`, every row of q has an entry of that size (bf16: 2^20) in a channel in which the keys are 0: what a
    scaled row loses of its other entries is then all the error there is.

    fp32: a score (size s, 1.4 here) is a sum of 2 x 128 products, each addition off by at most 2^-24 s and by 0.3 of
    that in the mean square: 16 x 0.3 x 1.4 x 2^-24 = 4e-7 of a probability; its exponential and the sums over the keys
    as much again: 1e-6 in all.  (Probabilities of 16 bits, 2^-16 at most, would give 2.5e-6; entries of q to 2^-25 of an
    outlier of 1e3 3e-5.)  bf16: beside the results' own rounding each probability is rounded, by itself and by half
    a step, 2^-8 of it, at most, so in a sum of independent terms the mean square grows by 2^-16 of the results' at most.
    With 16 rows a KV head or fewer it is off by 2^-16 at most, and so is the result but for its own rounding (1% of which
    is for the roundings that fall to the other side)."""
    from paper_2412_10418_amd import binding as bd
    rng = np.random.default_rng([case.B, case.n, 72])
    cache, lens, some, k, v = _filled(rng, case, fmt, quiet=5)
    q = 0.5 * torch.from_numpy(rng.standard_normal((case.B, case.n, case.H, case.hd), np.float32)).cuda()
    if outlier:
        size = outlier if kind == "f32" else 2.0 ** 20
        q[..., 5] = size * torch.from_numpy(rng.choice(np.float32([-1.7, -1, 1, 1.3]), q.shape[:3])).cuda()
    q = q.to(KIND[kind])
    parents = np.stack([random_tree(rng, case.n, 3) for _ in range(case.B)])
    out = _np(bd.cdsl_op_tree_attention(cache, q, _ints(lens), _ints(parents), max_len=case.longest))
    off, own, ref = [], [], []
    for i, b in enumerate(some):
        o, _, _ = attention(_np(q[b]).astype(np.float64), k[i][:lens[b] + case.n], v[i][:lens[b] + case.n], lens[b],
                            parents[b], case.hd ** -0.5)
        off.append((out[b] - o).ravel())
        own.append((_np(torch.from_numpy(o).to(KIND[kind])) - o).ravel())
        ref.append(o.ravel())
    off, own, ref = (rms(np.concatenate(x)) for x in (off, own, ref))
    print(f"{case.name} {kind} {fmt}: off by {off / ref:.3g} of the results, their own rounding {own / ref:.3g}", flush=True)
    if kind == "f32":
        assert off <= 1e-6 * ref
    elif case.kernel(kind, fmt).startswith("few1"):
        assert off <= 1.01 * own + 2.0 ** -16 * ref
    else:
        assert off ** 2 <= own ** 2 + (2.0 ** -8 * ref) ** 2


@pytest.mark.parametrize("V", [3001, 32768, 40001])
@pytest.mark.parametrize("v", [0.6995 / 0.9, 0.7005 / 0.9, 0.3995 / 0.9, 0.4005 / 0.9])
def test_what_is_left_of_a_draft_that_is_nearly_used_up(V, v):
    """Three siblings drawn without replacement leave 2^-45 of the draft, so that the rejected tokens' terms are 2^45 times
    what the target has left beside them; the draws are 5e-4 from a border."""
    p, q = np.zeros((1, 4, V), np.float32), np.zeros((1, 4, V), np.float32)
    for t, x in ((11, 0.4), (200, 0.1), (400, 0.3), (500, 0.2)):
        p[:, :, t] = x
    for t, x in ((10, 1 - 2.0 ** -24), (200, 2.0 ** -24 - 2.0 ** -45), (300, 2.0 ** -46)):
        q[:, :, t] = x
    tokens, parents = np.array([[0, 10, 200, 300]], np.int32), np.array([[-1, 0, 0, 0]], np.int32)
    _verify(p, q, tokens, parents, np.full((1, 4), 0.9, np.float32), np.full(1, v, np.float32), False)


@pytest.mark.parametrize("V", [300, 20000, 40001])
@pytest.mark.parametrize("at", [0, 17, 299])
@pytest.mark.parametrize("bad", [np.nan, -np.nan])
def test_a_nan_in_the_draft_row_of_a_rejection(V, at, bad):
    """It is in the sum of what is left: no token."""
    from paper_2412_10418_amd import binding as bd
    p, q = np.full((1, 2, V), 1 / V, np.float32), np.full((1, 2, V), 1 / (2 * V), np.float32)
    q[:, :, 5], q[0, 0, at] = 1, bad
    f = lambda x: torch.from_numpy(np.ascontiguousarray(x, np.float32)).cuda()  # noqa: E731
    path, m, tok = bd.cdsl_op_tree_accept(f(p), f(q), _ints([[0, 5]]), _ints([[-1, 0]]), f([[0.9, 0.9]]), f([0.5]))
    assert path.tolist() == [[0, -1]] and m.tolist() == [1] and tok.tolist() == [-1]


@pytest.mark.parametrize("V", [300, 20000, 40001])
@pytest.mark.parametrize("at", [0, 17, 299])
def test_infinities_of_a_rejection(V, at):
    """One in the target's row, or in both at the same token, is a sum that is not finite; one in the draft's alone leaves
    nothing of its token, and the draw is among the others."""
    from paper_2412_10418_amd import binding as bd
    f = lambda x: torch.from_numpy(np.ascontiguousarray(x, np.float32)).cuda()  # noqa: E731
    for pi, qi, none in ((np.inf, 0, True), (np.inf, np.inf, True), (0, np.inf, False)):
        p, q = np.full((1, 2, V), 1 / V, np.float32), np.full((1, 2, V), 1 / (2 * V), np.float32)
        q[:, :, 5], p[0, 0, at], q[0, 0, at] = 1, pi, qi
        path, m, tok = bd.cdsl_op_tree_accept(f(p), f(q), _ints([[0, 5]]), _ints([[-1, 0]]), f([[0.9, 0.9]]), f([0.0]))
        assert path.tolist() == [[0, -1]] and m.tolist() == [1]
        assert tok.tolist() == [-1 if none else 1 if at == 0 else 0]

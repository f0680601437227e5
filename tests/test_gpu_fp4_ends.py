"""Where the 4-bit cache and the pages' calls could go wrong by their size or their stream: pools whose pages begin past 2^32
bytes, pools without prompts, work on a stream beside the default one.  All comparisons are exact."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu


def _ints(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")


def _step(cache, layer, lens, K, V, q, path):
    """Rows written behind lens, attended to, read back, kept: all that a step gives."""
    from paper_2412_10418_amd import binding as bd
    n = K.shape[1] // 2
    bd.cdsl_op_kvq_write(cache, K[:, :n], V[:, :n], layer=layer)
    bd.cdsl_op_kvq_write(cache, K[:, n:], V[:, n:], start=lens, layer=layer)
    out = [bd.cdsl_op_tree_attention(cache, q[:, :rows].contiguous(), lens, max_len=n, layer=layer) for rows in (1, 5, q.shape[1])]
    out.extend(bd.cdsl_op_kvq_read(cache, 2 * n, layer=layer))
    bd.cdsl_op_kvq_keep(cache, lens, path, _ints([4] * cache.batch))
    return out + list(bd.cdsl_op_kvq_read(cache, n + 4, layer=layer))


def _inputs(rng, B, n, heads, hd):
    def of(*shape):
        return torch.from_numpy(rng.standard_normal(shape).astype(np.float32)).cuda()
    return of(B, 2 * n, heads, hd), of(B, 2 * n, heads, hd), of(B, 40, 2 * heads, hd), _ints(np.tile([0, 3, 9, 30] + [-1] * (n - 4), (B, 1)))


def test_pages_behind_four_gigabytes():
    """A pool of 130,000 pages of 34 KB: its last pages, in either layer, hold what a small pool's hold; a compaction brings
    them to its front, a copy to another pool."""
    from paper_2412_10418_amd import binding as bd
    rng = np.random.default_rng(11)
    B, n, heads, hd, pages = 3, 64, 8, 128, 130000
    assert 34 * hd * heads * pages > 2 ** 32
    far = bd.QuantCache(bd.QuantCache.empty(2, pages, heads, hd, fmt="mxfp4"), _ints(pages - 1 - rng.permutation(12).reshape(B, 4)), hd, "mxfp4")
    near = bd.QuantCache(bd.QuantCache.empty(2, 12, heads, hd, fmt="mxfp4"), _ints(rng.permutation(12).reshape(B, 4)), hd, "mxfp4")
    far.pool.zero_(), near.pool.zero_()
    lens = _ints([n] * B)
    for layer in (0, 1):
        args = _inputs(rng, B, n, heads, hd)
        for a, b in zip(_step(far, layer, lens, *args), _step(near, layer, lens, *args)):
            assert torch.equal(a, b)
    refs = torch.zeros(pages, dtype=torch.int32, device="cuda")
    refs[pages - 12:] = 1
    other = bd.QuantCache(bd.QuantCache.empty(2, 20, heads, hd, fmt="mxfp4"), _ints(np.arange(12).reshape(B, 4)), hd, "mxfp4")
    bd.cdsl_op_pages_copy(far, far.table.reshape(-1), other, other.table.reshape(-1))
    # and back to pages that lie far into the pool
    back = bd.QuantCache(far.pool, _ints(pages - 100 + np.arange(12).reshape(B, 4)), hd, "mxfp4")
    bd.cdsl_op_pages_copy(other, other.table.reshape(-1), back, back.table.reshape(-1))
    assert int(bd.cdsl_op_pages_compact(far, refs)) == 12
    assert sorted(far.table.reshape(-1).tolist()) == list(range(12)) and refs[:12].eq(1).all() and not refs[12:].any()
    for layer in (0, 1):
        for c in (far, other, back):
            for a, b in zip(bd.cdsl_op_kvq_read(c, 4 * 32, layer=layer), bd.cdsl_op_kvq_read(near, 4 * 32, layer=layer)):
                assert torch.equal(a, b)
    # a prompt that shares its last page takes the lowest free one, and its contents
    bd.cdsl_op_pages_fork(far, refs, _ints([2, 1, 2]))
    assert bd.cdsl_op_pages_reserve(far, refs, _ints([100, 128, 100]), _ints([5, 0, 1]), 5).tolist() == [5, 0, 1]
    assert far.table[0, 3] != far.table[2, 3] and torch.equal(far.table[0, :3], far.table[2, :3])
    K = bd.cdsl_op_kvq_read(far, 128, layer=1)[0]
    assert torch.equal(K[0], K[2]) and torch.equal(K[2], bd.cdsl_op_kvq_read(near, 128, layer=1)[0][2])


def test_a_pool_without_prompts():
    from paper_2412_10418_amd import binding as bd
    pool = bd.QuantCache.empty(2, 9, 1, 32, fmt="mxfp4")
    pool.copy_(torch.arange(pool.numel(), device="cuda").remainder(251).reshape(pool.shape))
    before = pool.clone()
    c = bd.QuantCache(pool, torch.empty((0, 4), dtype=torch.int32, device="cuda"), 32, "mxfp4")
    refs, none = _ints([0, 1, 0, 0, 2, 0, 0, 0, 1]), _ints(np.zeros(0))
    bd.cdsl_op_pages_fork(c, refs, none)
    bd.cdsl_op_pages_free(c, refs, none)
    assert bd.cdsl_op_pages_reserve(c, refs, none, none, 7).shape == (0,)
    assert int(bd.cdsl_op_pages_compact(c, refs)) == 3
    assert refs.tolist() == [1, 1, 2, 0, 0, 0, 0, 0, 0]
    assert torch.equal(pool[:, :3], before[:, [8, 1, 4]])


def test_a_stream_of_its_own():
    """All calls on a side stream, behind long work on it, while the default stream goes on: the results are those of the
    default stream."""
    from paper_2412_10418_amd import binding as bd
    rng = np.random.default_rng(12)
    B, n, heads, hd = 3, 64, 2, 64
    args = _inputs(rng, B, n, heads, hd)
    lens = _ints([n] * B)

    def run():
        c = bd.QuantCache(bd.QuantCache.empty(1, 40, heads, hd, fmt="mxfp4"), torch.full((B, 6), -1, dtype=torch.int32, device="cuda"), hd, "mxfp4")
        c.pool.zero_()
        refs = torch.zeros(40, dtype=torch.int32, device="cuda")
        got = [bd.cdsl_op_pages_reserve(c, refs, lens * 0, lens * 2, 2 * n)]
        got += _step(c, 0, lens, *args)
        bd.cdsl_op_pages_fork(c, refs, _ints([1, 1, 0]))
        got.append(bd.cdsl_op_pages_reserve(c, refs, lens + 9, lens, n))
        bd.cdsl_op_pages_free(c, refs, lens + 40)
        got.append(bd.cdsl_op_pages_compact(c, refs))
        return got + [c.table, refs] + list(bd.cdsl_op_kvq_read(c, 96))

    want = run()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        a = torch.ones(4096, 4096, device="cuda")
        for _ in range(20):
            a = a @ a * (1 / 4096)
        have = run()
    torch.zeros(1 << 20, device="cuda").add_(1)
    side.synchronize()
    assert len(want) == len(have) and all(torch.equal(x, y) for x, y in zip(want, have))

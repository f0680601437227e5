"""Pages that prompts share, on the GPU, against the entry-by-entry form of pages_ref.py: whole numbers and bytes, all exact."""
import numpy as np
import pytest
import torch

from pages_ref import Pages

pytestmark = pytest.mark.gpu


def _ints(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")


class Both:
    """A cache on the GPU and its plain form, taken through the same calls."""

    def __init__(self, rng, B, P, pages, layers=2, heads=1, hd=32, fmt="mxfp4"):
        from paper_2412_10418_amd import binding as bd
        self.bd = bd
        pool = bd.QuantCache.empty(layers, pages, heads, hd, fmt=fmt)
        pool.copy_(torch.from_numpy(rng.integers(0, 256, pool.shape, dtype=np.uint8)))
        self.cache = bd.QuantCache(pool, torch.full((B, P), -1, dtype=torch.int32, device="cuda"), hd, fmt)
        self.refs = torch.zeros(pages, dtype=torch.int32, device="cuda")
        self.ref = Pages(self.cache.table.cpu().numpy(), self.refs.cpu().numpy(), pool.cpu().numpy())

    def fork(self, parents):
        self.bd.cdsl_op_pages_fork(self.cache, self.refs, _ints(parents))
        self.ref.fork(parents)
        self.same("fork")

    def free(self, lens):
        self.bd.cdsl_op_pages_free(self.cache, self.refs, _ints(lens))
        self.ref.free(lens)
        self.same("free")

    def reserve(self, lens, count, most):
        got = self.bd.cdsl_op_pages_reserve(self.cache, self.refs, _ints(lens), _ints(count), most)
        want = self.ref.reserve(lens, count, most)
        self.same("reserve")
        assert np.array_equal(got.cpu().numpy(), want)
        return want

    def compact(self):
        used = self.bd.cdsl_op_pages_compact(self.cache, self.refs)
        assert int(used) == self.ref.compact()
        self.same("compact")

    def same(self, what):
        t, r = self.cache.table.cpu().numpy(), self.refs.cpu().numpy()
        assert np.array_equal(t, self.ref.table) and np.array_equal(r, self.ref.refs), what
        assert np.array_equal(r, np.bincount(t[(t >= 0) & (t < len(r))], minlength=len(r))), what
        assert np.array_equal(self.cache.pool.cpu().numpy(), self.ref.pool), what


@pytest.mark.parametrize("B,P,pages", [(1, 1, 1), (1, 4, 3), (3, 5, 40), (8, 6, 12), (17, 9, 60), (40, 3, 500), (5, 40, 90)])
def test_runs_of_calls(B, P, pages):
    """Prompts that grow, fork, end and shrink, in pools that run out among them; now and then the pool is compacted."""
    rng = np.random.default_rng([B, P, pages])
    x = Both(rng, B, P, pages)
    lens = np.zeros(B, int)
    for step in range(25):
        count = rng.integers(-1, 70, B)
        most = int(rng.integers(1, 70))
        got = x.reserve(lens, count, most)
        lens = lens + got
        if step % 3 == 0:
            parents = np.where(rng.random(B) < 0.5, np.arange(B), rng.integers(-2, B + 2, B))
            x.fork(parents)
            lens = np.array([lens[p] if 0 <= p < B else 0 for p in parents])
        if step % 4 == 1:
            lens = np.where(rng.random(B) < 0.4, lens * rng.random(B), lens).astype(int)
            x.free(lens)
        if step % 5 == 4:
            x.compact()


def test_ends_of_tables_and_lengths():
    """Lengths below 0, at and behind a page's end and the table's; counts of 0 and beyond max_count."""
    rng = np.random.default_rng(1)
    x = Both(rng, 12, 3, 100)
    x.reserve([0] * 12, [96, 1, 31, 32, 33, 64, 65, 0, -5, 1000, 2 ** 31 - 1, 7], 96)
    x.fork([0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0])
    x.reserve([-1, -2 ** 31, 1, 31, 32, 33, 63, 64, 95, 96, 97, 2 ** 31 - 1], [1, 5, 31, 1, 1, 31, 2, 32, 1, 1, 1, 2 ** 31 - 1], 40)
    x.free([-1, -2 ** 31, 1, 31, 32, 33, 64, 65, 95, 96, 97, 2 ** 31 - 1])
    x.reserve([0] * 12, [3] * 12, 0)
    x.compact()


def test_the_first_that_leaves_keeps_the_page():
    """Four prompts on one page, all of which write: the first keeps it, three copies.  If one of them does not write, four
    minus one copies and it stays with that one.  If pages run out, nobody keeps it."""
    rng = np.random.default_rng(2)
    x = Both(rng, 4, 2, 9)
    x.reserve([0, 0, 0, 0], [0, 10, 0, 0], 10)
    x.fork([1, 1, 1, 1])
    page = int(x.cache.table[1, 0])
    x.reserve([10] * 4, [1] * 4, 1)
    assert int(x.cache.table[0, 0]) == page and len(set(x.cache.table[:, 0].tolist())) == 4
    x.fork([1, 1, 1, 1])
    page = int(x.cache.table[1, 0])
    assert x.reserve([10] * 4, [1, 1, 0, 1], 1).tolist() == [1, 1, 0, 1]
    assert int(x.cache.table[2, 0]) == page
    x = Both(rng, 4, 2, 3)
    x.reserve([0] * 4, [10, 0, 0, 0], 10)
    x.fork([0] * 4)
    assert x.reserve([10] * 4, [5] * 4, 8).tolist() == [0, 5, 5, 0]       # two free pages: the first does not keep the page
    x.fork([0, 1, 2, -1])          # the last holds nothing: the page is the first one's again
    assert x.reserve([10] * 4, [5, 5, 5, 0], 8).tolist() == [5, 5, 5, 0]


@pytest.mark.parametrize("B,P,pages,T", [(600, 7, 9000, 100), (513, 20, 8193, 640), (512, 33, 20000, 1030), (2000, 2, 1024, 33), (3, 3000, 10000, 96000)])
def test_many_prompts_and_pages(B, P, pages, T):
    """More entries and pages than the plan takes at once, tables that fork over two launches, free pages that end."""
    rng = np.random.default_rng([B, P])
    x = Both(rng, B, P, pages, layers=1)
    lens = np.zeros(B, int)
    got = x.reserve(lens, rng.integers(0, T + 1, B), T)
    x.fork(np.where(rng.random(B) < 0.7, np.arange(B), rng.integers(0, B, B)))
    lens = np.maximum(got - 40, 0)
    x.reserve(lens, rng.integers(0, T + 1, B), T)
    lens = lens // 2
    x.free(lens)
    x.compact()
    x.reserve(lens, np.full(B, 1), 1)


@pytest.mark.parametrize("fmt,heads,hd,layers", [("mxfp4", 1, 32, 3), ("mxfp4", 8, 128, 2), ("mxfp4", 3, 64, 5), ("int8", 32, 128, 2), ("e4m3", 5, 64, 1)])
def test_contents_of_every_format(fmt, heads, hd, layers):
    """Pages of one piece and of many, copied whole in all layers."""
    rng = np.random.default_rng([heads, hd])
    x = Both(rng, 6, 4, 30, layers, heads, hd, fmt)
    x.reserve([0] * 6, [70, 0, 0, 40, 0, 0], 70)
    x.fork([0, 0, 0, 3, 3, 3])
    x.reserve([70, 70, 66, 40, 33, 40], [9] * 6, 9)
    x.free([0, 70, 0, 40, 0, 40])
    x.compact()


def test_entries_that_are_no_pages():
    """Ids outside the pool hold nothing: they are passed on by a fork, replaced by a reserve, and given back as -1."""
    rng = np.random.default_rng(3)
    x = Both(rng, 3, 3, 20)
    x.reserve([0, 0, 0], [96, 40, 0], 96)
    for at, v in (((0, 1), 20), ((0, 2), 2 ** 31 - 1), ((1, 0), -2 ** 31), ((2, 0), -7)):
        old = int(x.cache.table[at])
        if 0 <= old < 20:
            x.refs[old] -= 1
            x.ref.refs[old] -= 1
        x.cache.table[at] = v
        x.ref.table[at] = v
    x.fork([0, 0, 2])
    x.compact()
    x.reserve([40, 64, 0], [40, 1, 1], 40)
    x.free([32, 0, 0])


def test_pages_between_pools():
    from paper_2412_10418_amd import binding as bd
    rng = np.random.default_rng(4)
    x, y = Both(rng, 1, 1, 50, 3, 2, 64), Both(rng, 2, 5, 90, 3, 2, 64)
    src, dst = rng.permutation(50)[:40], rng.permutation(90)[:40]
    src[3], src[4], dst[5], dst[6] = -1, 50, 90, -2 ** 31
    bd.cdsl_op_pages_copy(x.cache, _ints(src), y.cache, _ints(dst))
    want = y.ref.pool
    for s, d in zip(src, dst):
        if 0 <= s < 50 and 0 <= d < 90:
            want[:, d] = x.ref.pool[:, s]
    assert np.array_equal(y.cache.pool.cpu().numpy(), want) and np.array_equal(x.cache.pool.cpu().numpy(), x.ref.pool)
    # within a pool, a page onto itself among them
    bd.cdsl_op_pages_copy(x.cache, _ints([1, 2, 9]), x.cache, _ints([11, 2, 19]))
    x.ref.pool[:, [11, 19]] = x.ref.pool[:, [1, 9]]
    x.same("copy")
    bd.cdsl_op_pages_copy(x.cache, _ints([]), x.cache, _ints([]))
    with pytest.raises(ValueError):
        bd.cdsl_op_pages_copy(x.cache, _ints([1]), y.cache, _ints([1, 2]))
    with pytest.raises(bd.CDSLError):
        bd.cdsl_op_pages_copy(x.cache, _ints([1]), Both(rng, 1, 1, 50, 3, 2, 32).cache, _ints([1]))


def test_a_captured_step_is_replayed():
    """Fork, reserve and free in one graph, replayed over lengths and parents that change, beside eager work."""
    from paper_2412_10418_amd import binding as bd
    rng = np.random.default_rng(5)
    B, P, pages = 12, 6, 60
    x = Both(rng, B, P, pages)
    lens = np.full(B, 20)
    x.reserve(np.zeros(B, int), lens, 20)
    parents, at, count, left = (_ints(np.zeros(B)) for _ in range(4))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        bd.cdsl_op_pages_fork(x.cache, x.refs, parents)
        got = bd.cdsl_op_pages_reserve(x.cache, x.refs, at, count, 50)
        bd.cdsl_op_pages_free(x.cache, x.refs, left)
        used = bd.cdsl_op_pages_compact(x.cache, x.refs)
    x.same("after the capture, which runs nothing")
    for step in range(6):
        p = rng.integers(0, B, B)
        lens = lens[p]
        n = rng.integers(0, 51, B)
        parents.copy_(_ints(p))
        at.copy_(_ints(lens))
        count.copy_(_ints(n))
        left.copy_(_ints(lens + n // 2))
        graph.replay()
        torch.cuda.synchronize()
        x.ref.fork(p)
        g = x.ref.reserve(lens, n, 50)
        x.ref.free(lens + n // 2)
        u = x.ref.compact()
        assert np.array_equal(got.cpu().numpy(), g) and int(used) == u
        x.same(f"replay {step}")
        lens = np.minimum(lens + n // 2, lens + g)
        torch.zeros(1000, device="cuda").sum().item()


@pytest.mark.parametrize("fmt", ["mxfp4", "int8"])
def test_beams_serve_as_if_each_had_its_own_cache(fmt):
    """Two prompts x three beams: forked from the chosen beam, room reserved, tokens written, attended and kept, the rest given
    back, the pool compacted.  Each beam's attention is, bit for bit, that of a cache of its own with the same rows."""
    from paper_2412_10418_amd import binding as bd
    rng = np.random.default_rng(6)
    B, k, heads, hd, n = 6, 3, 2, 64, 5
    x = Both(rng, B, 8, 60, 1, heads, hd, fmt)
    own = Both(rng, B, 8, 60, 1, heads, hd, fmt)
    lens = np.array([75, 0, 0, 40, 0, 0])

    def rows(T):
        return [torch.from_numpy(rng.standard_normal((B, T, heads, hd)).astype(np.float32)).cuda() for _ in range(2)]

    x.reserve(np.zeros(B, int), lens, 75)
    K, V = rows(75)
    bd.cdsl_op_kvq_write(x.cache, K, V, count=_ints(lens))
    history = [(K[b, :lens[b]], V[b, :lens[b]]) for b in range(B)]
    for step in range(4):
        chosen = np.repeat([rng.integers(0, k) if step else 0, k + (rng.integers(0, k) if step else 0)], k)
        bd.cdsl_op_pages_fork(x.cache, x.refs, _ints(chosen))
        lens = lens[chosen]
        got = bd.cdsl_op_pages_reserve(x.cache, x.refs, _ints(lens), _ints(np.full(B, n)), n)
        assert (got == n).all()
        K, V = rows(n)
        bd.cdsl_op_kvq_write(x.cache, K, V, start=_ints(lens))
        q = torch.from_numpy(rng.standard_normal((B, n, 4, hd)).astype(np.float32)).cuda()
        out = bd.cdsl_op_tree_attention(x.cache, q, _ints(lens), max_len=int(lens.max()))
        history = [history[c] for c in chosen]
        # the same rows in caches that share nothing
        own.bd.cdsl_op_pages_free(own.cache, own.refs, _ints(np.zeros(B)))
        assert (bd.cdsl_op_pages_reserve(own.cache, own.refs, _ints(np.zeros(B)), _ints(lens + n), int(lens.max()) + n).cpu().numpy() == lens + n).all()
        for b in range(B):
            history[b] = (torch.cat([history[b][0], K[b]]), torch.cat([history[b][1], V[b]]))
        T = max(len(h[0]) for h in history)
        full = [torch.stack([torch.nn.functional.pad(h[i], (0, 0, 0, 0, 0, T - len(h[i]))) for h in history]).contiguous() for i in (0, 1)]
        bd.cdsl_op_kvq_write(own.cache, *full, count=_ints(lens + n))
        assert torch.equal(out, bd.cdsl_op_tree_attention(own.cache, q, _ints(lens), max_len=int(lens.max())))
        # three of the five tokens are kept, the pages behind them given back
        path = np.tile([0, 2, 3, -1, -1], (B, 1))
        new = bd.cdsl_op_kvq_keep(x.cache, _ints(lens), _ints(path), _ints(np.full(B, 3)))
        history = [(torch.cat([h[0][:L], h[0][[L, L + 2, L + 3]]]), torch.cat([h[1][:L], h[1][[L, L + 2, L + 3]]])) for h, L in zip(history, lens)]
        bd.cdsl_op_pages_free(x.cache, x.refs, new)
        used = int(bd.cdsl_op_pages_compact(x.cache, x.refs))
        assert int((x.refs > 0).sum()) == used and not (x.refs[used:] > 0).any()
        lens = lens + 3

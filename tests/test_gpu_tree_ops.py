"""The operators around a drafted tree on the GPU, against plain 64-bit forms
(tree_ref.py): the 8-bit cache (exact: codes and scales are defined to the
bit), tree attention (bounds derived in tree_ref.tolerance), the verification
(tokens and nodes exact), the kept path (bytes), and a run of them together."""
import numpy as np
import pytest
import torch

from tree_ref import attention, close, paged, quantised, random_tree, tolerance, walk

pytestmark = pytest.mark.gpu

FMTS = ("int8", "e4m3")
KIND = {"f32": torch.float32, "bf16": torch.bfloat16}


def _rows(rng, shape, kind):
    x = rng.standard_normal(shape, np.float32) * np.exp(rng.standard_normal(shape[-1], np.float32))
    return torch.from_numpy(x.astype(np.float32)).cuda().to(KIND[kind])


def _ints(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")


def _np(t):
    return t.float().cpu().numpy()


def _same(x, y):
    """The same bits (leftovers of a page may well be NaN)."""
    return torch.equal(x.contiguous().view(torch.uint8), y.contiguous().view(torch.uint8))


# ---------------------------------------------------------------------------
# the cache
# ---------------------------------------------------------------------------
@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("B,T,heads,hd,start", [(1, 1, 1, 32, 0), (1, 1, 8, 128, 95), (3, 33, 2, 64, 31), (2, 64, 5, 128, 32),
                                                (4, 70, 3, 32, 7), (2, 257, 4, 128, 0), (5, 31, 1, 64, 1)])
def test_rows_read_back_as_their_codes_say(fmt, kind, B, T, heads, hd, start):
    """Bitwise: the value is the fp32 product of a code and a scale that the definition gives exactly.  Slots outside the
    runs keep their bytes."""
    from paper_2412_10418_amd import binding as bd
    rng = np.random.default_rng([T, heads, hd, start])
    cache = paged(rng, 2, B, start + T + 9, heads, hd, fmt)
    K, V = _rows(rng, (B, T, heads, hd), kind), _rows(rng, (B, T, heads, hd), kind)
    at = _ints(start + rng.integers(0, 9, B))
    count = _ints(np.minimum(T, np.maximum(0, T - rng.integers(-2, T + 2, B))))
    count[0] = T
    before = cache.pool.clone()
    bd.cdsl_op_kvq_write(cache, K, V, start=at, count=count, layer=1)
    k, v = bd.cdsl_op_kvq_read(cache, T, start=at, count=count, layer=1)
    for b in range(B):
        m = int(count[b])
        for got, x in ((k, K), (v, V)):
            assert np.array_equal(_np(got[b, :m]), quantised(_np(x[b, :m]), fmt))
            assert not got[b, m:].any()
    # bytes: nothing but the run's codes and scales changed
    assert torch.equal(cache.pool[0], before[0])
    changed = int((cache.pool[1] != before[1]).sum())
    assert changed <= int(count.sum()) * heads * (2 * hd + 8)
    kb, vb = bd.cdsl_op_kvq_read(cache, T, start=at, count=count, layer=1, dtype=torch.bfloat16)
    assert torch.equal(kb, k.bfloat16()) and torch.equal(vb, v.bfloat16())


@pytest.mark.parametrize("fmt", FMTS)
def test_writes_leave_their_neighbours(fmt):
    """A run that starts and ends inside pages: the slots before and behind it read as before, whatever the order of the
    writes."""
    from paper_2412_10418_amd import binding as bd
    rng = np.random.default_rng(5)
    cache = paged(rng, 1, 1, 128, 3, 64, fmt)
    K, V = _rows(rng, (1, 128, 3, 64), "f32"), _rows(rng, (1, 128, 3, 64), "f32")
    for a, b in ((40, 41), (100, 128), (0, 40), (41, 43), (97, 100), (43, 97)):
        bd.cdsl_op_kvq_write(cache, K[:, a:b], V[:, a:b], start=_ints([a]))
    k, v = bd.cdsl_op_kvq_read(cache, 128)
    assert np.array_equal(_np(k), quantised(_np(K), fmt)) and np.array_equal(_np(v), quantised(_np(V), fmt))


@pytest.mark.parametrize("fmt", FMTS)
def test_rows_at_the_borders_of_their_codes(fmt):
    """Ties of the rounding, zeros, the largest and the smallest numbers, rows with a NaN or an infinity."""
    from paper_2412_10418_amd import binding as bd
    rng = np.random.default_rng(6)
    x = np.zeros((14, 32), np.float32)
    x[0, :] = np.arange(32) / 2                       # max 15.5
    x[1, :] = np.arange(-16, 16) + 0.5
    x[1, 0] = 127.0                                   # scale 1: every entry is a tie
    x[2, :] = np.nextafter(np.arange(32) + np.float32(0.5), np.float32(1e9) * (-1) ** np.arange(32), dtype=np.float32)
    x[2, 0] = -127.0                                  # one step off the ties
    x[3, :] = 2.0 ** -np.arange(32.0)                 # down to subnormal e4m3 codes
    x[3, 0] = 448.0
    x[4, :] = (1 + np.arange(32) / 16) * 16           # e4m3 ties between its 3-bit steps
    x[4, 0] = 448.0
    x[5, 3] = np.float32(np.nextafter(np.float32(448), np.float32(1e9)))   # the next scale
    x[6, :] = np.float32(3.4e38) * rng.uniform(-1, 1, 32)
    x[7, :] = np.float32(1e-38) * rng.uniform(-1, 1, 32)
    x[8, :] = np.float32(1e-44)
    x[10, 5] = np.nan
    x[11, 7] = -np.inf
    x[12, :] = 127 * 1.2345 * np.float32(2.0) ** -100
    x[12, 1:] = x[12, 0] / 127 * (np.arange(31) + np.float32(0.5)).astype(np.float32)
    x[13, :] = rng.uniform(-1, 1, 32)
    cache = paged(rng, 1, 1, 14, 1, 32, fmt)
    t = torch.from_numpy(x).cuda().view(1, 14, 1, 32)
    bd.cdsl_op_kvq_write(cache, t, t.flip(1).contiguous())
    k, v = bd.cdsl_op_kvq_read(cache, 14)
    assert np.array_equal(_np(k)[0, :, 0], quantised(x, fmt), equal_nan=True)
    assert np.array_equal(_np(v)[0, ::-1, 0], quantised(x, fmt), equal_nan=True)


@pytest.mark.parametrize("fmt", FMTS)
def test_many_values_are_rounded_exactly(fmt):
    """2^22 values of unlike rows (fp32 quotients land on the wrong side of a tie about once in 10^5)."""
    from paper_2412_10418_amd import binding as bd
    rng = np.random.default_rng(7)
    cache = paged(rng, 1, 1, 4096, 8, 128, fmt)
    x = _rows(rng, (1, 4096, 8, 128), "f32") * torch.exp2(torch.randint(-30, 30, (1, 4096, 8, 1), device="cuda").float())
    bd.cdsl_op_kvq_write(cache, x, -x)
    k, v = bd.cdsl_op_kvq_read(cache, 4096)
    ref = quantised(_np(x), fmt)
    assert np.array_equal(_np(k), ref) and np.array_equal(_np(v), -ref)


def test_strided_rows_and_slices_of_a_projection():
    """K and V as slices of one [B, T, (H + 2 heads) hd] projection, tokens of another order, one row for all prompts."""
    from paper_2412_10418_amd import binding as bd
    rng = np.random.default_rng(8)
    B, T, H, heads, hd = 3, 37, 4, 2, 64
    qkv = _rows(rng, (B, T, (H + 2 * heads), hd), "bf16")
    K, V = qkv[:, :, H:H + heads], qkv[:, :, H + heads:]
    cache = paged(rng, 1, B, T, heads, hd, "int8")
    bd.cdsl_op_kvq_write(cache, K, V)
    k, v = bd.cdsl_op_kvq_read(cache, T)
    assert np.array_equal(_np(k), quantised(_np(K), "int8")) and np.array_equal(_np(v), quantised(_np(V), "int8"))
    one = _rows(rng, (1, T, heads, hd), "f32").expand(B, T, heads, hd)
    swapped = _rows(rng, (T, B, heads, hd), "f32").transpose(0, 1)
    bd.cdsl_op_kvq_write(cache, one, swapped)
    k, v = bd.cdsl_op_kvq_read(cache, T)
    assert np.array_equal(_np(k), quantised(_np(one), "int8")) and np.array_equal(_np(v), quantised(_np(swapped), "int8"))


def test_positions_without_a_page_are_left_alone():
    """Bad page ids, positions beyond the table and below 0: not written, NaN when read."""
    from paper_2412_10418_amd import binding as bd
    rng = np.random.default_rng(9)
    cache = paged(rng, 1, 3, 96, 2, 32, "int8", fill=0)
    table = cache.table.clone()
    table[0, 1], table[1, 2], table[2, 0] = -1, cache.pool.shape[1], 2 ** 31 - 1
    bad = bd.QuantCache(cache.pool, table, 32, "int8")
    x = _rows(rng, (3, 130, 2, 32), "f32")
    at = _ints([0, -7, 5])
    bd.cdsl_op_kvq_write(bad, x, x, start=at)
    k, _ = bd.cdsl_op_kvq_read(bad, 130, start=at)
    pos = np.arange(130)[None, :] + np.array([0, -7, 5])[:, None]
    ok = (pos >= 0) & (pos < 96)
    ids = table.cpu().numpy()
    live = np.take_along_axis(ids, np.clip(pos // 32, 0, 2), 1)
    ok &= (live >= 0) & (live < cache.pool.shape[1])
    ref = quantised(_np(x), "int8")
    assert np.array_equal(_np(k)[ok], ref[ok]) and np.isnan(_np(k)[~ok]).all()
    # pages that no position has stay as they were
    used = set(live[ok].tolist())
    for p in range(cache.pool.shape[1]):
        if p not in used:
            assert not cache.pool[0, p].any()


# ---------------------------------------------------------------------------
# attention
# ---------------------------------------------------------------------------
def _filled(rng, B, lens, n, heads, hd, fmt, layers=1, kind="f32", spare=2):
    from paper_2412_10418_amd import binding as bd
    T = max(lens) + n
    cache = paged(rng, layers, B, T, heads, hd, fmt, spare=spare)
    K, V = _rows(rng, (B, T, heads, hd), kind), _rows(rng, (B, T, heads, hd), kind)
    count = _ints([l + n for l in lens])
    bd.cdsl_op_kvq_write(cache, K, V, count=count, layer=layers - 1)
    k, v = bd.cdsl_op_kvq_read(cache, T, count=count, layer=layers - 1)
    return cache, _np(k).astype(np.float64), _np(v).astype(np.float64)


def _check(out, q, k, v, lens, parents, nodes, scale, what):
    bf16 = out.dtype == torch.bfloat16
    got, x = _np(out), _np(q).astype(np.float64)
    for b, L in enumerate(lens):
        m = nodes[b]
        if m == 0:
            continue
        par = None if parents is None else parents[b]
        ref, mag, top = attention(x[b, :m], k[b][:L + m], v[b][:L + m], L, par, scale)
        close(got[b, :m], ref, tolerance(mag, top, x.shape[-1], L + m, bf16), f"{what} prompt {b}")


CASES = [  # B, n, H, heads, hd, lens
    (1, 1, 1, 1, 32, [0]), (1, 1, 8, 1, 128, [31]), (3, 1, 8, 8, 64, [0, 1, 700]), (2, 5, 6, 2, 128, [32, 33]),
    (2, 17, 4, 4, 64, [63, 0]), (3, 51, 4, 4, 128, [256, 0, 95]), (2, 65, 8, 2, 128, [100, 1]), (1, 130, 10, 2, 32, [77]),
    (2, 33, 12, 4, 64, [5, 1000]), (1, 300, 2, 1, 128, [40]),
]


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("shape", ["tree", "causal", "star", "forest"])
@pytest.mark.parametrize("case", CASES, ids=[f"{c[0]}x{c[1]}-{c[2]}.{c[3]}x{c[4]}" for c in CASES])
def test_tree_attention(fmt, kind, shape, case):
    from paper_2412_10418_amd import binding as bd
    B, n, H, heads, hd, lens = case
    rng = np.random.default_rng([n, H, hd, len(shape)])
    cache, k, v = _filled(rng, B, lens, n, heads, hd, fmt)
    q = (1.5 * _rows(rng, (B, n, H, hd), "f32")).to(KIND[kind])
    parents = None if shape == "causal" else np.stack([random_tree(rng, n, 3, shape) for _ in range(B)])
    out = bd.cdsl_op_tree_attention(cache, q, _ints(lens), None if parents is None else _ints(parents), max_len=max(lens))
    _check(out, q, k, v, lens, parents, [n] * B, hd ** -0.5, f"{shape} {fmt} {kind}")


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("B,n,H,heads,hd,L", [(1, 1, 8, 1, 128, 5000), (2, 3, 4, 2, 64, 3111), (1, 7, 40, 8, 32, 2049),
                                              (1, 40, 8, 1, 128, 1500)])
def test_split_keys(kind, B, n, H, heads, hd, L):
    """Contexts long enough to be split over workgroups, ragged so that a split of a short prompt is empty; the bound on
    the lengths changes the split, not the result beyond rounding."""
    from paper_2412_10418_amd import binding as bd
    rng = np.random.default_rng([n, H, L])
    lens = [L] + [int(rng.integers(0, 40)) for _ in range(B - 1)]
    assert bd.lib().cdsl_op_tree_attention_workspace(B, n, H, heads, hd, L) > 0
    cache, k, v = _filled(rng, B, lens, n, heads, hd, "int8")
    q = _rows(rng, (B, n, H, hd), "f32").to(KIND[kind])
    parents = np.stack([random_tree(rng, n, 3) for _ in range(B)])
    for bound in (L, 0, 100 * L, 700):
        out = bd.cdsl_op_tree_attention(cache, q, _ints(lens), _ints(parents), max_len=bound)
        _check(out, q, k, v, lens, parents, [n] * B, hd ** -0.5, f"bound {bound} {kind}")


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("B,n,H,heads,hd,L", [(2, 1, 8, 1, 32, 40000), (31, 1, 8, 2, 64, 2600), (64, 2, 8, 2, 32, 9000),
                                              (65, 1, 2, 1, 32, 2100), (3, 70, 2, 1, 128, 3000), (9, 40, 4, 2, 64, 1200),
                                              (12, 65, 32, 8, 32, 4200), (40, 1, 16, 8, 32, 4200),
                                              (8, 17, 32, 8, 32, 4200), (8, 30, 32, 8, 64, 4200)])
def test_a_long_prompt_among_short_ones(kind, B, n, H, heads, hd, L):
    """The key splits go to the prompts by their lengths: one long, others short or empty, without nodes, or past what
    the table holds (NaN); rows behind a prompt's nodes stay as they were."""
    from paper_2412_10418_amd import binding as bd
    rng = np.random.default_rng([B, n, L])
    lens = rng.integers(0, 70, B).tolist()
    at = int(rng.integers(0, B))
    lens[at] = L
    nodes = np.full(B, n)
    if B > 2:
        lens[(at + 1) % B], nodes[(at + 1) % B] = 0, 0
        lens[(at + 2) % B] = 0
    assert bd.lib().cdsl_op_tree_attention_workspace(B, n, H, heads, hd, L) > 0
    cache, k, v = _filled(rng, B, lens, n, heads, hd, "int8")
    q = _rows(rng, (B, n, H, hd), "f32").to(KIND[kind])
    parents = np.stack([random_tree(rng, n, 3) for _ in range(B)])
    long = lens.copy()
    over = (at + 3) % B if B > 3 else None
    if over is not None:
        long[over] = cache.table.shape[1] * 32 - n + 1
    for given in (lens, long):
        out = torch.full_like(q, 7.0)
        bd.cdsl_op_tree_attention(cache, q, _ints(given), _ints(parents), n_nodes=_ints(nodes), max_len=L, out=out)
        some = [b for b in sorted({0, at, (at + 1) % B, (at + 2) % B, B - 1}) if given[b] == lens[b]]
        _check(out[some], q[some], k[some], v[some], [lens[b] for b in some], parents[some], nodes[some].tolist(),
               hd ** -0.5, f"{kind} at {at}")
        for b in range(B):
            assert bool((out[b, nodes[b]:] == 7).all())
            if given[b] == lens[b]:
                assert torch.isfinite(out[b, :nodes[b]]).all()
            else:
                assert torch.isnan(out[b, :nodes[b]]).all()


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("hd,n,causal", [(128, 64, False), (64, 61, True), (32, 64, False)])
def test_batches_that_fill_the_chip(fmt, kind, hd, n, causal):
    """Enough rows for waves of two row tiles (the last tiles part empty at 61 nodes), prompts of unlike lengths and node
    counts in no order."""
    from paper_2412_10418_amd import binding as bd
    rng = np.random.default_rng([hd, n])
    B, H, heads = 97, 16, 8
    lens = rng.integers(0, 140, B).tolist()
    lens[5], lens[90] = 0, 150
    nodes = rng.integers(1, n + 1, B)
    nodes[[5, 50, 90]] = n
    cache, k, v = _filled(rng, B, lens, n, heads, hd, fmt)
    q = (1.5 * _rows(rng, (B, n, H, hd), "f32")).to(KIND[kind])
    parents = None if causal else np.stack([random_tree(rng, n, 3) for _ in range(B)])
    out = bd.cdsl_op_tree_attention(cache, q, _ints(lens), None if causal else _ints(parents), n_nodes=_ints(nodes),
                                    max_len=max(lens))
    some = [0, 5, 17, 50, 90, 96]
    _check(out[some], q[some], k[some], v[some], [lens[b] for b in some], None if causal else parents[some],
           nodes[some].tolist(), hd ** -0.5, f"{fmt} {kind}")
    for b in range(B):
        assert torch.isfinite(out[b, :nodes[b]]).all() and not out[b, nodes[b]:].any()


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("causal", [True, False])
def test_long_chunks_that_fill_the_chip(kind, causal):
    """Several row groups a prompt, the last one part empty, and prompts whose nodes end in any of them."""
    from paper_2412_10418_amd import binding as bd
    rng = np.random.default_rng([61, int(causal)])
    B, n, H, heads, hd = 25, 62, 64, 8, 32
    lens = rng.integers(0, 200, B).tolist()
    nodes = rng.integers(0, n + 1, B)
    nodes[[0, 7]] = n, 1
    cache, k, v = _filled(rng, B, lens, n, heads, hd, "int8")
    q = _rows(rng, (B, n, H, hd), "f32").to(KIND[kind])
    parents = None if causal else np.stack([random_tree(rng, n, 3) for _ in range(B)])
    out = torch.full_like(q, 7.0)
    bd.cdsl_op_tree_attention(cache, q, _ints(lens), None if causal else _ints(parents), n_nodes=_ints(nodes),
                              max_len=200, out=out)
    _check(out, q, k, v, lens, parents, nodes.tolist(), hd ** -0.5, kind)
    for b in range(B):
        assert bool((out[b, nodes[b]:] == 7).all())


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("L", [3, 2500])
def test_nodes_that_a_prompt_lacks(kind, L):
    """Fewer nodes than n, none, and counts out of range: the rows behind are left as they were."""
    from paper_2412_10418_amd import binding as bd
    rng = np.random.default_rng(21)
    B, n, H, heads, hd = 5, 19, 4, 2, 64
    lens = [L, 0, 40, 7, 1]
    cache, k, v = _filled(rng, B, lens, n, heads, hd, "e4m3")
    q = _rows(rng, (B, n, H, hd), "f32").to(KIND[kind])
    parents = np.stack([random_tree(rng, n, 3) for _ in range(B)])
    out = torch.full_like(q, 7.0)
    nodes = [19, 0, 1, -4, 1000]
    bd.cdsl_op_tree_attention(cache, q, _ints(lens), _ints(parents), n_nodes=_ints(nodes), max_len=L, out=out)
    nodes = [19, 0, 1, 0, 19]
    _check(out, q, k, v, lens, parents, nodes, hd ** -0.5, kind)
    for b, m in enumerate(nodes):
        assert bool((out[b, m:] == 7).all())


@pytest.mark.parametrize("fmt", FMTS)
def test_unwritten_slots_do_not_matter(fmt):
    """Every byte outside the written slots is a NaN code and a NaN scale, then zero: the same bits."""
    from paper_2412_10418_amd import binding as bd
    rng = np.random.default_rng(22)
    B, n, H, heads, hd = 2, 9, 4, 2, 128
    outs = []
    for fill in (0xFF, 0x7F, 0):
        r = np.random.default_rng(23)
        cache = paged(r, 1, B, 90, heads, hd, fmt, fill=fill)
        K, V = _rows(r, (B, 79, heads, hd), "f32"), _rows(r, (B, 79, heads, hd), "f32")
        bd.cdsl_op_kvq_write(cache, K, V, count=_ints([79, 12]))
        q = _rows(r, (B, n, H, hd), "f32")
        outs.append(bd.cdsl_op_tree_attention(cache, q, _ints([70, 3]), _ints(np.stack([random_tree(r, n, 3)] * B))))
    assert torch.isfinite(outs[0]).all() and torch.equal(outs[0], outs[1]) and torch.equal(outs[0], outs[2])


def test_nan_rows_and_missing_pages_reach_the_rows_that_see_them():
    from paper_2412_10418_amd import binding as bd
    rng = np.random.default_rng(24)
    B, n, H, heads, hd = 4, 6, 4, 2, 64
    lens = [40, 40, 40, 33]
    T = 40 + n
    cache = paged(rng, 1, B, T, heads, hd, "int8")
    K, V = _rows(rng, (B, T, heads, hd), "f32"), _rows(rng, (B, T, heads, hd), "f32")
    K[0, 42, 1, 3] = float("nan")            # node 2 of prompt 0, KV head 1
    V[1, 44, 0, 5] = float("inf")            # node 4 of prompt 1, KV head 0
    bd.cdsl_op_kvq_write(cache, K, V)
    table = cache.table.clone()
    table[2, 0] = cache.pool.shape[1]        # prompt 2 lacks its first page
    cut = bd.QuantCache(cache.pool, table[:, :2].contiguous(), hd, "int8")
    parents = np.array([[-1, 0, 0, 2, 1, 4]] * B, np.int32)
    q = _rows(rng, (B, n, H, hd), "f32")
    for kind in (torch.float32, torch.bfloat16):
        out = bd.cdsl_op_tree_attention(cut, q.to(kind), _ints(lens), _ints(parents))
        nan = torch.isnan(out).cpu().numpy()
        expect = np.zeros_like(nan)
        expect[0, [2, 3], 2:] = True         # node 2 and its child 3; query heads of KV head 1
        expect[1, [4, 5], :2] = True
        expect[2] = True
        assert np.array_equal(nan, expect)
    # a table that cannot hold lens + nodes: NaN, whatever the lengths say
    out = bd.cdsl_op_tree_attention(cut, q, _ints([59, 58, 2 ** 31 - 1, -9]), _ints(parents))
    assert torch.isnan(out[0]).all() and torch.isnan(out[2]).all() and not torch.isnan(out[3]).any()
    long = bd.cdsl_op_tree_attention(cut, q, _ints([59, 58, 2 ** 31 - 1, -9]), _ints(parents), max_len=30000)
    assert torch.isnan(long[0]).all() and torch.isnan(long[2]).all() and not torch.isnan(long[3]).any()


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("B,n,H,heads", [(1, 14, 2, 2), (2, 24, 2, 2), (2, 24, 8, 2), (100, 64, 16, 8)])
def test_a_missing_page_spares_the_rows_that_do_not_see_it(fmt, kind, B, n, H, heads):
    """A star whose nodes from 12 on lie on a page that the pool does not have, in a pool of NaN codes and scales."""
    from paper_2412_10418_amd import binding as bd
    rng = np.random.default_rng([n, H])
    L, hd = 20, 64
    cache = paged(rng, 1, B, L + n, heads, hd, fmt, fill=0xFF)
    table = cache.table.clone()
    table[table == 0] = next(i for i in range(cache.pool.shape[1]) if i not in set(table.flatten().tolist()))
    cache = bd.QuantCache(cache.pool, table, hd, fmt)
    K, V = _rows(rng, (B, L + n, heads, hd), kind), _rows(rng, (B, L + n, heads, hd), kind)
    bd.cdsl_op_kvq_write(cache, K, V)
    k, v = bd.cdsl_op_kvq_read(cache, L + n)
    k, v = _np(k).astype(np.float64), _np(v).astype(np.float64)
    q = _rows(rng, (B, n, H, hd), kind)
    parents = np.stack([random_tree(rng, n, 3, "star")] * B)
    whole = table[:, 1].clone()
    for missing in (-1, cache.pool.shape[1]):
        table[:, 1] = missing
        out = bd.cdsl_op_tree_attention(cache, q, _ints([L] * B), _ints(parents))
        on_it = torch.arange(n, device="cuda").add(L).floor_divide(32) == 1
        assert torch.isnan(out[:, on_it]).all() and torch.isfinite(out[:, ~on_it]).all()
        _check(out[:2, :12], q[:2, :12], k, v, [L] * min(B, 2), parents[:, :12], [12] * min(B, 2), hd ** -0.5, f"{fmt} {kind}")
    table[:, 1] = whole
    assert torch.isfinite(bd.cdsl_op_tree_attention(cache, q, _ints([L] * B), _ints(parents))).all()


@pytest.mark.parametrize("kind", ["f32", "bf16"])
def test_scores_far_apart_and_scales(kind):
    """Sharp softmaxes (scores to some hundreds), a zero and a negative scale, and values of unlike sizes."""
    from paper_2412_10418_amd import binding as bd
    rng = np.random.default_rng(25)
    B, n, H, heads, hd, lens = 2, 7, 4, 2, 128, [300, 64]
    cache, k, v = _filled(rng, B, lens, n, heads, hd, "int8")
    q = (6 * _rows(rng, (B, n, H, hd), "f32")).to(KIND[kind])
    parents = np.stack([random_tree(rng, n, 2) for _ in range(B)])
    for scale in (0.3, 0.0, -0.05):
        out = bd.cdsl_op_tree_attention(cache, q, _ints(lens), _ints(parents), scale=scale)
        _check(out, q, k, v, lens, parents, [n] * B, scale, f"scale {scale}")


def test_queries_of_a_projection_and_layers():
    from paper_2412_10418_amd import binding as bd
    rng = np.random.default_rng(26)
    B, n, H, heads, hd, lens = 3, 11, 6, 2, 64, [9, 0, 70]
    cache, k, v = _filled(rng, B, lens, n, heads, hd, "e4m3", layers=3)
    qkv = _rows(rng, (B, n, H + 2 * heads, hd), "f32")
    q = qkv[:, :, :H]
    assert not q.is_contiguous()
    out = bd.cdsl_op_tree_attention(cache, q, _ints(lens), layer=2)
    _check(out, q, k, v, lens, None, [n] * B, hd ** -0.5, "slice")
    assert torch.equal(out, bd.cdsl_op_tree_attention(cache, q.contiguous(), _ints(lens), layer=2))


def test_prompts_that_share_their_pages():
    """Beams over one prompt: the same prefix pages in every table, own pages for the nodes."""
    from paper_2412_10418_amd import binding as bd
    rng = np.random.default_rng(27)
    B, n, H, heads, hd, L = 4, 5, 4, 2, 64, 96
    cache = paged(rng, 1, B, L + 32, heads, hd, "int8")
    table = cache.table.clone()
    table[:, :3] = table[0, :3]
    c = bd.QuantCache(cache.pool, table, hd, "int8")
    one = bd.QuantCache(cache.pool, table[:1].contiguous(), hd, "int8")
    pre = _rows(rng, (1, L, heads, hd), "f32")
    bd.cdsl_op_kvq_write(one, pre, -pre)
    own = _rows(rng, (B, n, heads, hd), "f32")
    bd.cdsl_op_kvq_write(c, own, own, start=_ints([L] * B))
    k, v = (_np(t).astype(np.float64) for t in bd.cdsl_op_kvq_read(c, L + n))
    q = _rows(rng, (B, n, H, hd), "f32")
    out = bd.cdsl_op_tree_attention(c, q, _ints([L] * B))
    _check(out, q, k, v, [L] * B, None, [n] * B, hd ** -0.5, "shared")


def test_pages_beyond_four_gigabytes():
    """Byte offsets past 2^32 in the pool, in every operator that follows a page."""
    from paper_2412_10418_amd import binding as bd
    rng = np.random.default_rng(28)
    heads, hd, pages = 8, 128, 70000                      # 4.73 GB a layer
    pool = bd.QuantCache.empty(1, pages, heads, hd)
    ids = np.array([[69999, 3, 65000], [64000, 69998, 0]], np.int32)
    cache = bd.QuantCache(pool, _ints(ids), hd, "int8")
    x = _rows(rng, (2, 90, heads, hd), "f32")
    bd.cdsl_op_kvq_write(cache, x, -x)
    k, v = bd.cdsl_op_kvq_read(cache, 90)
    ref = quantised(_np(x), "int8")
    assert np.array_equal(_np(k), ref) and np.array_equal(_np(v), -ref)
    q = _rows(rng, (2, 4, 16, hd), "f32")
    out = bd.cdsl_op_tree_attention(cache, q, _ints([86, 80]))
    kk, vv = _np(k).astype(np.float64), _np(v).astype(np.float64)
    _check(out, q, kk, vv, [86, 80], None, [4, 4], hd ** -0.5, "far pages")
    new = bd.cdsl_op_kvq_keep(cache, _ints([60, 62]), _ints([[0, 5, 7], [2, 3, 9]]), _ints([3, 2]))
    k2, _ = bd.cdsl_op_kvq_read(cache, 90)
    assert new.tolist() == [63, 64]
    assert torch.equal(k2[0, 61:63], k[0, [65, 67]]) and torch.equal(k2[1, 62:64], k[1, [64, 65]])


# ---------------------------------------------------------------------------
# verification
# ---------------------------------------------------------------------------
def _verify(p, q, tokens, parents, u, v, replace, n_nodes=None):
    from paper_2412_10418_amd import binding as bd
    f = lambda x: torch.from_numpy(np.ascontiguousarray(x, np.float32)).cuda()  # noqa: E731
    path, m, tok = bd.cdsl_op_tree_accept(f(p), f(q), _ints(tokens), _ints(parents), f(u), f(v), replace=replace,
                                          n_nodes=None if n_nodes is None else _ints(n_nodes))
    path, m, tok = path.cpu().numpy(), m.tolist(), tok.tolist()
    for b in range(p.shape[0]):
        nb = p.shape[1] if n_nodes is None else min(max(n_nodes[b], 1), p.shape[1])
        ref, x = walk(p[b, :nb], q[b, :nb], tokens[b], parents[b], u[b], v[b], replace)
        assert path[b, :m[b]].tolist() == ref and (path[b, m[b]:] == -1).all(), (b, path[b], ref)
        assert tok[b] == x, (b, tok[b], x)
    return path, m, tok


def _soft(z):
    e = np.exp(z - z.max(-1, keepdims=True))
    return (e / e.sum(-1, keepdims=True)).astype(np.float32)


@pytest.mark.parametrize("replace", [True, False])
@pytest.mark.parametrize("B,n,V,width", [(1, 1, 1, 1), (3, 2, 2, 1), (8, 16, 5, 3), (5, 40, 1000, 4), (16, 51, 4097, 5),
                                         (4, 130, 32000, 3), (2, 33, 50257, 8), (1, 9, 128256, 4), (3, 512, 257, 2)])
def test_trees_are_verified(replace, B, n, V, width):
    """Random trees, drafts near and far from the target, peaked and flat rows: every node and token as the definition
    gives them in 64 bits."""
    rng = np.random.default_rng([n, V, width])
    for near in (0.3, 2.0):
        z = rng.standard_normal((B, n, V)) * rng.choice([0.1, 3.0], (B, n, 1))
        p, q = _soft(z), _soft(z + near * rng.standard_normal((B, n, V)))
        parents = np.stack([random_tree(rng, n, width) for _ in range(B)])
        tokens = np.empty((B, n), np.int32)
        for b in range(B):
            for j in range(n):
                tokens[b, j] = rng.choice(V, p=q[b, max(0, parents[b, j])].astype(np.float64) / q[b, max(0, parents[b, j])].astype(np.float64).sum())
        u, v = rng.random((B, n), np.float32), rng.random(B, np.float32)
        path, m, _ = _verify(p, q, tokens, parents, u, v, replace)
        print(f"near {near}: {np.mean(m):.2f} nodes a path", flush=True)


@pytest.mark.parametrize("V", [3001, 40001])
@pytest.mark.parametrize("replace", [True, False])
def test_many_siblings_are_rejected(replace, V):
    """A star of 40 siblings whose target mass is elsewhere: a chain of rejections, with duplicates among the tokens (more
    sums than long rows have launches for)."""
    rng = np.random.default_rng(31)
    B, n = 6, 41
    z = rng.standard_normal((B, n, V))
    p, q = _soft(2 * z), _soft(-z)
    tokens = np.argsort(-q[:, 0], -1)[:, :n].astype(np.int32)
    tokens[:, 5] = tokens[:, 4]
    tokens[:, 9] = tokens[:, 4]
    parents = np.stack([random_tree(rng, n, 2, "star")] * B)
    u = np.full((B, n), 0.999, np.float32)
    _, m, _ = _verify(p, q, tokens, parents, u, rng.random(B, np.float32), replace)
    assert min(m) == 1


@pytest.mark.parametrize("replace", [True, False])
@pytest.mark.parametrize("B,V", [(33, 33001), (17, 40000), (16, 70000)])
def test_batches_of_long_rows(replace, B, V):
    """Walks of unlike lengths in one batch: prompts that are over in the first launch, others that reject seven
    siblings and go on from the eighth."""
    rng = np.random.default_rng([B, V])
    n = 10
    z = rng.standard_normal((B, n, V), np.float32)
    p, q = _soft(z + 2 * (rng.random((B, 1, 1)) < 0.5) * rng.standard_normal((B, n, V), np.float32)), _soft(z)
    parents = np.tile(np.array([-1] + [0] * 8 + [8], np.int32), (B, 1))
    tokens = np.argsort(-q[:, 0], -1)[:, :n].astype(np.int32)
    u = np.where(rng.random((B, n)) < 0.3, 0.2, 0.999).astype(np.float32)
    u[::3, 1:8], u[::3, 8] = 0.9999, 0.0
    _, m, _ = _verify(p, q, tokens, parents, u, rng.random(B, np.float32), replace)
    print(f"paths of {sorted(set(m))} nodes", flush=True)


@pytest.mark.parametrize("V", [70, 33001])
@pytest.mark.parametrize("replace", [True, False])
def test_rows_at_the_borders_of_the_walk(replace, V):
    """Equal rows, one-hot rows, rows without mass, draws at 0 and just below 1, tokens and parents out of range."""
    rng = np.random.default_rng(32)
    n = 6
    p = np.zeros((9, n, V), np.float32)
    q = np.zeros((9, n, V), np.float32)
    base = _soft(rng.standard_normal((n, V)))
    tokens = np.tile(rng.permutation(V)[:n].astype(np.int32), (9, 1))
    parents = np.tile(np.array([-1, 0, 0, 1, 1, 0], np.int32), (9, 1))
    u = np.full((9, n), 0.5, np.float32)
    v = np.full(9, 0.5, np.float32)
    p[0], q[0] = base, base                                    # equal: the first child is always kept
    p[1], q[1] = base, 0                                       # a draft without mass
    q[1, :, 3] = 1
    tokens[1, 1:3] = 3                                         # drafted from a point: kept by its probability
    u[1] = 0.9999
    p[2, :, 7], q[2] = 1, base                                 # a point of the target
    tokens[2, 2] = 7
    p[3], q[3] = base, base
    p[3, 0], q[3, 0] = 0, 0                                    # no mass at all
    p[4], q[4] = base * 0.5, base                              # no mass above the draft's: argmax p
    u[4], tokens[4, 1] = 1 - 2.0 ** -24, np.argmax(base[0])
    p[5], q[5], v[5] = base, base[::-1], 0.0
    u[5] = 0.9999
    p[6], q[6], v[6] = base, base[::-1], 1 - 2.0 ** -24
    p[6, :, -20:] = 0                                          # the last ids have no mass
    u[6] = 0.9999
    p[7], q[7] = base, base
    tokens[7, 1], tokens[7, 2], tokens[7, 3] = -1, V, 2 ** 31 - 1
    parents[7] = [5, 0, 0, 0, 99, -7]
    p[8], q[8], u[8] = base, base[::-1], 0.0                   # u = 0 keeps any child with mass
    _verify(p, q, tokens, parents, u, v, replace)


@pytest.mark.parametrize("V", [300, 70000])
def test_sums_that_are_not_finite(V):
    from paper_2412_10418_amd import binding as bd
    for bad in (np.nan, np.inf, -np.nan):
        p = np.full((1, 2, V), 1 / V, np.float32)
        p[0, 0, 17] = bad
        q = np.full_like(p, 1 / V)
        path, m, tok = bd.cdsl_op_tree_accept(torch.from_numpy(p).cuda(), torch.from_numpy(q).cuda(), _ints([[0, 17]]),
                                              _ints([[-1, -1]]), torch.zeros(1, 2, device="cuda"),
                                              torch.full((1,), 0.5, device="cuda"))
        assert path.tolist() == [[0, -1]] and m.tolist() == [1] and tok.tolist() == [-1]


def test_prompts_with_fewer_nodes():
    rng = np.random.default_rng(33)
    B, n, V = 5, 20, 500
    z = rng.standard_normal((B, n, V))
    p, q = _soft(z), _soft(z)
    parents = np.stack([random_tree(rng, n, 2, "chain")] * B)
    tokens = rng.integers(0, V, (B, n)).astype(np.int32)
    nodes = [20, 1, 0, 7, 99]
    _, m, _ = _verify(p, q, tokens, parents, np.zeros((B, n), np.float32), rng.random(B, np.float32), True, nodes)
    assert m == [20, 1, 1, 7, 20]


def test_draws_follow_the_target():
    """What the walk emits first has the target's distribution: 40000 walks over one node of eight tokens with two drafted
    children.  A frequency's deviation is sqrt(f (1 - f) / 40000), 0.0025 at most; five of them."""
    rng = np.random.default_rng(34)
    N, V = 40000, 8
    p, q = _soft(rng.standard_normal(V)), _soft(rng.standard_normal(V))
    for replace in (True, False):
        drawn = np.empty((N, 2), np.int64)
        drawn[:, 0] = rng.choice(V, N, p=q.astype(np.float64) / q.astype(np.float64).sum())
        for i in range(N):
            w = q.astype(np.float64).copy()
            if not replace:
                w[drawn[i, 0]] = 0
            drawn[i, 1] = np.searchsorted(np.cumsum(w / w.sum()), rng.random(), side="right")
        tokens = np.concatenate([np.zeros((N, 1)), drawn], 1).astype(np.int32)
        from paper_2412_10418_amd import binding as bd
        f = lambda x: torch.from_numpy(np.ascontiguousarray(x, np.float32)).cuda()  # noqa: E731
        rows = lambda x: f(np.broadcast_to(x, (N, 3, V)))  # noqa: E731
        path, m, tok = bd.cdsl_op_tree_accept(rows(p), rows(q), _ints(tokens), _ints(np.tile([-1, 0, 0], (N, 1))),
                                              f(rng.random((N, 3))), f(rng.random(N)), replace=replace)
        path, m, tok = path.cpu().numpy(), m.cpu().numpy(), tok.cpu().numpy()
        first = np.where(m > 1, tokens[np.arange(N), np.maximum(path[:, 1], 0)], tok)
        freq = np.bincount(first, minlength=V) / N
        assert np.abs(freq - p).max() < 0.0125, (freq, p)


# ---------------------------------------------------------------------------
# the kept path, and all of it together
# ---------------------------------------------------------------------------
@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("B,n,heads,hd,layers", [(1, 1, 1, 32, 1), (3, 12, 2, 64, 2), (2, 70, 5, 128, 3), (4, 200, 1, 32, 2)])
def test_kept_paths_move_to_the_front(fmt, B, n, heads, hd, layers):
    """Every byte of the pool: the kept entries at their new slots, everything else as before."""
    from paper_2412_10418_amd import binding as bd
    rng = np.random.default_rng([n, hd])
    lens = rng.integers(0, 70, B)
    cache = paged(rng, layers, B, 70 + n, heads, hd, fmt)
    x = _rows(rng, (B, 70 + n, heads, hd), "f32")
    for l in range(layers):
        bd.cdsl_op_kvq_write(cache, x + l, x - l, layer=l)
    m = rng.integers(1, n + 1, B)
    path = np.full((B, n), -1, np.int32)
    for b in range(B):
        path[b, :m[b]] = np.sort(rng.permutation(n)[:m[b]])
    before = [[t.clone() for t in bd.cdsl_op_kvq_read(cache, 70 + n, layer=l)] for l in range(layers)]
    new = bd.cdsl_op_kvq_keep(cache, _ints(lens), _ints(path), _ints(m))
    assert new.tolist() == (lens + m).tolist()
    for l in range(layers):
        for got, old in zip(bd.cdsl_op_kvq_read(cache, 70 + n, layer=l), before[l]):
            want = old.clone()
            for b in range(B):
                want[b, lens[b]:lens[b] + m[b]] = old[b, lens[b] + path[b, :m[b]]]
            assert torch.equal(got, want)


def test_paths_without_pages_and_counts_out_of_range():
    from paper_2412_10418_amd import binding as bd
    rng = np.random.default_rng(41)
    cache = paged(rng, 1, 4, 64, 2, 32, "int8")
    x = _rows(rng, (4, 64, 2, 32), "f32")
    bd.cdsl_op_kvq_write(cache, x, x)
    k, _ = bd.cdsl_op_kvq_read(cache, 64)
    table = cache.table.clone()
    table[1, 1] = -5
    bad = bd.QuantCache(cache.pool, table, 32, "int8")
    path = _ints([[0, 2, 3], [0, 1, 2], [0, 512, -9], [1, 2, 99]])
    new = bd.cdsl_op_kvq_keep(bad, _ints([62, 30, 10, 3]), path, _ints([9, 3, 3, -1]))
    assert new.tolist() == [65, 33, 13, 3]
    got, _ = bd.cdsl_op_kvq_read(cache, 64)
    assert torch.equal(got, k)          # nothing could move: beyond the table, no page, no node of a tree, a count below 0


def _step(cache, state, layers):
    """One verification step over a tree as a user makes it."""
    from paper_2412_10418_amd import binding as bd
    outs = []
    for l in range(layers):
        bd.cdsl_op_kvq_write(cache, state["K"][l], state["V"][l], start=state["lens"], count=state["nodes"], layer=l)
        outs.append(bd.cdsl_op_tree_attention(cache, state["q"][l], state["lens"], state["parents"],
                                              n_nodes=state["nodes"], max_len=state["bound"], layer=l))
    path, m, tok = bd.cdsl_op_tree_accept(state["p"], state["d"], state["tokens"], state["parents"], state["u"],
                                          state["v"], n_nodes=state["nodes"])
    new = bd.cdsl_op_kvq_keep(cache, state["lens"], path, m)
    return outs, path, m, tok, new


def _state(rng, B, n, H, heads, hd, V, layers, lens, kind, bound):
    z = rng.standard_normal((B, n, V))
    parents = np.stack([random_tree(rng, n, 3) for _ in range(B)])
    f = lambda x: torch.from_numpy(np.ascontiguousarray(x, np.float32)).cuda()  # noqa: E731
    return dict(K=[_rows(rng, (B, n, heads, hd), kind) for _ in range(layers)],
                V=[_rows(rng, (B, n, heads, hd), kind) for _ in range(layers)],
                q=[_rows(rng, (B, n, H, hd), kind) for _ in range(layers)], lens=_ints(lens),
                nodes=_ints(rng.integers(1, n + 1, B)), parents=_ints(parents), p=f(_soft(z)),
                d=f(_soft(z + 0.5 * rng.standard_normal(z.shape))), tokens=_ints(rng.integers(0, V, (B, n))),
                u=f(0.3 * rng.random((B, n))), v=f(rng.random(B)), bound=bound)


@pytest.mark.parametrize("fmt,kind", [("int8", "f32"), ("e4m3", "bf16")])
def test_steps_over_drafted_trees(fmt, kind):
    """Prompts written, then five steps (write, attend in two layers, verify, keep): lengths, kept entries and every
    attention against a cache of the same values held in float64."""
    from paper_2412_10418_amd import binding as bd
    rng = np.random.default_rng(51)
    B, n, H, heads, hd, V, layers = 3, 13, 6, 2, 64, 200, 2
    lens = np.array([45, 0, 17])
    cache = paged(rng, layers, B, 150, heads, hd, fmt)
    held = [[[None] * B for _ in range(2)] for _ in range(layers)]
    for l in range(layers):
        K, Vv = _rows(rng, (B, 45, heads, hd), kind), _rows(rng, (B, 45, heads, hd), kind)
        bd.cdsl_op_kvq_write(cache, K, Vv, count=_ints(lens), layer=l)
        for i, x in enumerate((K, Vv)):
            for b in range(B):
                held[l][i][b] = quantised(_np(x[b, :lens[b]]), fmt).astype(np.float64)
    for step in range(5):
        s = _state(rng, B, n, H, heads, hd, V, layers, lens, kind, int(lens.max()))
        outs, path, m, tok, new = _step(cache, s, layers)
        m, path, nodes = m.tolist(), path.cpu().numpy(), s["nodes"].tolist()
        for b in range(B):
            ref, x = walk(_np(s["p"][b, :nodes[b]]), _np(s["d"][b, :nodes[b]]), s["tokens"][b].tolist(),
                          s["parents"][b].tolist(), _np(s["u"][b]), float(s["v"][b]), True)
            assert path[b, :m[b]].tolist() == ref and int(tok[b]) == x
        for l in range(layers):
            kv = [[np.concatenate([held[l][i][b], quantised(_np(s[w][l][b, :nodes[b]]), fmt).astype(np.float64)])
                   for b in range(B)] for i, w in enumerate("KV")]
            _check(outs[l], s["q"][l], kv[0], kv[1], lens.tolist(), s["parents"].cpu().numpy(), nodes, hd ** -0.5,
                   f"step {step} layer {l}")
            for i in range(2):
                for b in range(B):
                    held[l][i][b] = np.concatenate([held[l][i][b], kv[i][b][lens[b] + path[b, :m[b]]]])
        lens = lens + np.array(m)
        assert new.tolist() == lens.tolist()
    for l in range(layers):
        k, v = bd.cdsl_op_kvq_read(cache, int(lens.max()), count=_ints(lens), layer=l)
        for b in range(B):
            assert np.array_equal(_np(k[b, :lens[b]]), held[l][0][b].astype(np.float32))
            assert np.array_equal(_np(v[b, :lens[b]]), held[l][1][b].astype(np.float32))


@pytest.mark.parametrize("bound,V", [(60, 300), (4000, 40000)])
def test_captured_steps_replay_as_they_run(bound, V):
    """Two graphs of a step over one cache, replayed in turn on new inputs with eager steps of another cache between
    them: every replay gives the eager result's bits."""
    rng = np.random.default_rng(52)
    B, n, H, heads, hd, layers = 2, 9, 4, 2, 64, 2
    a, e, other = (paged(np.random.default_rng(53), layers, B, 128 + bound, heads, hd, "int8") for _ in range(3))
    states = [_state(rng, B, n, H, heads, hd, V, layers, [40, 11], "f32", bound) for _ in range(2)]
    _step(other, states[0], layers)
    torch.cuda.synchronize()
    graphs = []
    for s in states:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            got = _step(a, s, layers)
        graphs.append((g, got))
    for turn in range(4):
        for s, (g, got) in zip(states, graphs):
            fresh = _state(rng, B, n, H, heads, hd, V, layers, rng.integers(0, 60, B), "f32", bound)
            for k, x in fresh.items():
                if isinstance(x, list):
                    for dst, src in zip(s[k], x):
                        dst.copy_(src)
                elif torch.is_tensor(x):
                    s[k].copy_(x)
            g.replay()
            _step(other, s, layers)
            want = _step(e, s, layers)
            torch.cuda.synchronize()
            for x, y in zip(list(got[0]) + list(got[1:]), list(want[0]) + list(want[1:])):
                assert _same(x, y)
            assert torch.equal(a.pool, e.pool)


def test_steps_on_two_streams_at_once():
    """Independent caches on two streams give what they give alone."""
    rng = np.random.default_rng(54)
    B, n, H, heads, hd, V, layers = 2, 21, 8, 2, 128, 5000, 2
    sets = [_state(rng, B, n, H, heads, hd, V, layers, [700, 300], "bf16", 700) for _ in range(2)]
    alone = []
    for s in sets:
        c = paged(np.random.default_rng(55), layers, B, 800, heads, hd, "e4m3", fill=0)
        alone.append((_step(c, s, layers), c))
    torch.cuda.synchronize()
    caches = [paged(np.random.default_rng(55), layers, B, 800, heads, hd, "e4m3", fill=0) for _ in sets]
    streams = [torch.cuda.Stream() for _ in sets]
    torch.cuda.synchronize()
    got = [None, None]
    for _ in range(3):
        for i, s in enumerate(sets):
            with torch.cuda.stream(streams[i]):
                caches[i].pool.zero_()
                got[i] = _step(caches[i], s, layers)
    torch.cuda.synchronize()
    for i in range(2):
        for x, y in zip(list(got[i][0]) + list(got[i][1:]), list(alone[i][0][0]) + list(alone[i][0][1:])):
            assert _same(x, y)
        assert torch.equal(caches[i].pool, alone[i][1].pool)

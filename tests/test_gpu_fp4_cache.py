"""The 4-bit cache on the GPU: rows written and read back, the bytes of its units, and the kept path, all exact (codes and
scales are defined to the bit), against the 64-bit forms of fp4_ref.py."""
import numpy as np
import pytest
import torch

from fp4_ref import coded, paged, places, quantised, token_bytes

pytestmark = pytest.mark.gpu

KIND = {"f32": torch.float32, "bf16": torch.bfloat16}


def _rows(rng, shape, kind):
    x = rng.standard_normal(shape, np.float32) * np.exp(rng.standard_normal(shape[-1], np.float32))
    return torch.from_numpy(x.astype(np.float32)).cuda().to(KIND[kind])


def _ints(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")


def _np(t):
    return t.float().cpu().numpy()


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("B,T,heads,hd,start", [(1, 1, 1, 32, 0), (1, 1, 8, 128, 95), (3, 33, 2, 64, 31), (2, 64, 5, 128, 32),
                                                (4, 70, 3, 32, 7), (2, 257, 4, 128, 0), (5, 31, 1, 64, 1), (1, 2050, 1, 128, 33)])
def test_rows_read_back_as_their_codes_say(kind, B, T, heads, hd, start):
    """Bitwise; and the pool's bytes are the definition's, those outside the runs as they were."""
    from paper_2412_10418_amd import binding as bd
    rng = np.random.default_rng([T, heads, hd, start])
    cache = paged(rng, 2, B, start + T + 9, heads, hd)
    K, V = _rows(rng, (B, T, heads, hd), kind), _rows(rng, (B, T, heads, hd), kind)
    first = start + rng.integers(0, 9, B)
    count = np.minimum(T, np.maximum(0, T - rng.integers(-2, T + 2, B)))
    count[0] = T
    want = cache.pool.cpu().numpy()
    bd.cdsl_op_kvq_write(cache, K, V, start=_ints(first), count=_ints(count), layer=1)
    k, v = bd.cdsl_op_kvq_read(cache, T, start=_ints(first), count=_ints(count), layer=1)
    table, at = cache.table.cpu().numpy(), places(hd)
    for b in range(B):
        m = count[b]
        for got, x in ((k, K), (v, V)):
            assert np.array_equal(_np(got[b, :m]), quantised(_np(x[b, :m])))
            assert not got[b, m:].any()
        byte = token_bytes(_np(K[b, :m]), _np(V[b, :m]))
        for t in range(m):
            p = first[b] + t
            for h in range(heads):
                want[1, table[b, p // 32], h, at[p % 32]] = byte[t, h]
    assert np.array_equal(cache.pool.cpu().numpy(), want)
    kb, vb = bd.cdsl_op_kvq_read(cache, T, start=_ints(first), count=_ints(count), layer=1, dtype=torch.bfloat16)
    assert torch.equal(kb, k.bfloat16()) and torch.equal(vb, v.bfloat16())
    assert torch.equal(kb.float(), k)          # code times a power of two: exact in bf16


def test_writes_leave_their_neighbours():
    from paper_2412_10418_amd import binding as bd
    rng = np.random.default_rng(5)
    for hd in (32, 64, 128):
        cache = paged(rng, 1, 1, 128, 3, hd)
        K, V = _rows(rng, (1, 128, 3, hd), "f32"), _rows(rng, (1, 128, 3, hd), "f32")
        for a, b in ((40, 41), (100, 128), (0, 40), (41, 43), (97, 100), (43, 97)):
            bd.cdsl_op_kvq_write(cache, K[:, a:b], V[:, a:b], start=_ints([a]))
        k, v = bd.cdsl_op_kvq_read(cache, 128)
        assert np.array_equal(_np(k), quantised(_np(K))) and np.array_equal(_np(v), quantised(_np(V)))


def _borders():
    x = np.zeros((20, 32), np.float32)
    ties = np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0], np.float32)
    x[0, :7], x[0, 7] = ties, 6.0
    x[1, :7], x[1, 7] = -ties, 6.0
    x[2, :7], x[2, 7] = np.nextafter(ties, np.float32(9)), 6.0
    x[3, :7], x[3, 7] = np.nextafter(ties, np.float32(0)), -6.0
    x[4, :8] = [0, 0.5, 1, 1.5, 2, 3, 4, 6]
    x[5, 3] = np.nextafter(np.float32(6), np.float32(9))            # the next scale
    x[6, :] = -0.0
    x[7, :] = 2.0 ** -np.arange(32.0)
    x[8, :] = np.float32(3.4e38) * np.linspace(-1, 1, 32)           # the largest numbers: at most 6 * 2^125
    x[9, :] = np.float32(1.5 * 2.0 ** 127)
    x[10, :] = np.float32(2.0 ** -126) * np.linspace(-1, 1, 32)     # the smallest: below half a step of 2^-125
    x[11, :] = np.float32(1e-44)
    x[12, :] = np.float32(2.0 ** -125) * np.linspace(-8, 8, 32)
    x[13, 5] = np.nan
    x[14, 7] = -np.inf
    x[15, :] = np.float32(2.0 ** -127)                              # half of the smallest code's value: a tie, to 0
    x[16, :] = np.nextafter(np.float32(2.0 ** -127), np.float32(1))
    x[17, :] = np.arange(32) / 4
    x[18, :] = np.arange(32) / 4 * np.float32(2.0) ** 100
    x[19, 0] = np.nextafter(np.float32(1.5 * 2.0 ** 127), np.float32(0))
    return x


def test_rows_at_the_borders_of_their_codes():
    """Ties, zeros of both signs, the largest and the smallest numbers, rows with a NaN or an infinity."""
    from paper_2412_10418_amd import binding as bd
    rng = np.random.default_rng(6)
    x = _borders()
    n = len(x)
    cache = paged(rng, 1, 1, n, 1, 32)
    t = torch.from_numpy(x).cuda().view(1, n, 1, 32)
    bd.cdsl_op_kvq_write(cache, t, t.flip(1).contiguous())
    k, v = bd.cdsl_op_kvq_read(cache, n)
    want = quantised(x)
    assert np.array_equal(_np(k)[0, :, 0], want, equal_nan=True) and np.array_equal(_np(v)[0, ::-1, 0], want, equal_nan=True)
    assert np.array_equal(np.signbit(_np(k)[0, :13, 0]), np.signbit(want[:13]))


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("kind", ["f32", "bf16"])
def test_blocks_have_their_own_scales_and_a_nan_takes_the_row(hd, kind):
    from paper_2412_10418_amd import binding as bd
    rng = np.random.default_rng(hd)
    x = _rows(rng, (1, 70, 2, hd), kind)
    x = (x.view(1, 70, 2, hd // 32, 32) * torch.exp2(torch.randint(-60, 60, (1, 70, 2, hd // 32, 1), device="cuda").float())).view(1, 70, 2, hd).to(KIND[kind])
    x[0, 3, 0, hd - 1] = float("nan")
    x[0, 40, 1, 0] = float("inf")
    x[0, 69, 0, 33] = float("-inf")
    cache = paged(rng, 1, 1, 70, 2, hd)
    bd.cdsl_op_kvq_write(cache, x, x)
    k, v = bd.cdsl_op_kvq_read(cache, 70)
    want = quantised(_np(x))
    assert np.isnan(want).sum() == 3 * hd
    assert np.array_equal(_np(k), want, equal_nan=True) and np.array_equal(_np(v), want, equal_nan=True)


def test_strided_rows_and_pages_that_do_not_exist():
    """Views with gaps between prompts and tokens; ids outside the pool and positions outside the table are not written and
    read as NaN."""
    from paper_2412_10418_amd import binding as bd
    rng = np.random.default_rng(8)
    cache = paged(rng, 1, 2, 96, 2, 64)
    big = _rows(rng, (2, 80, 3, 2, 64), "bf16")
    K, V = big[:, :, 0], big[:, :, 2]
    cache.table[0, 1] = -1
    cache.table[1, 2] = cache.pool.shape[1]
    before = cache.pool.clone()
    start = _ints([20, -5])
    bd.cdsl_op_kvq_write(cache, K, V, start=start)
    k, v = bd.cdsl_op_kvq_read(cache, 80, start=start)
    for got, x in ((k, K), (v, V)):
        want = quantised(_np(x))
        pos = np.stack([20 + np.arange(80), -5 + np.arange(80)])
        want[0, (pos[0] >= 32) & (pos[0] < 64)] = np.nan
        want[0, pos[0] >= 96] = np.nan
        want[1, (pos[1] < 0) | (pos[1] >= 64)] = np.nan
        assert np.array_equal(_np(got), want, equal_nan=True)
    kept = [p for p in range(cache.pool.shape[1]) if p not in cache.table.flatten().tolist()]
    assert torch.equal(cache.pool[:, kept], before[:, kept])


@pytest.mark.parametrize("hd,heads,layers", [(32, 3, 2), (64, 2, 3), (128, 8, 2)])
@pytest.mark.parametrize("n,most", [(1, 1), (9, 4), (51, 8), (200, 40)])
def test_kept_entries_move_and_the_rest_stays(hd, heads, layers, n, most):
    from paper_2412_10418_amd import binding as bd
    rng = np.random.default_rng([hd, n])
    B = 5
    lens = np.array([0, 1, 30, 95, 256])
    cache = paged(rng, layers, B, 256 + n, heads, hd)
    path = np.full((B, n), -1)
    count = np.zeros(B, int)
    for b in range(B):
        count[b] = rng.integers(0, most + 1) if b else most
        path[b, :count[b]] = np.sort(rng.permutation(n)[:count[b]])
    want, table, at = cache.pool.cpu().numpy(), cache.table.cpu().numpy(), places(hd)
    for b in range(B):
        for i in range(count[b]):
            s, d = lens[b] + path[b, i], lens[b] + i
            want[:, table[b, d // 32], :, at[d % 32][:, None, None]] = want[:, table[b, s // 32], :, at[s % 32][:, None, None]]
    new = bd.cdsl_op_kvq_keep(cache, _ints(lens), _ints(path), _ints(count))
    assert np.array_equal(new.cpu().numpy(), lens + count)
    assert np.array_equal(cache.pool.cpu().numpy(), want)


def test_kept_entries_without_a_page_stay():
    from paper_2412_10418_amd import binding as bd
    rng = np.random.default_rng(9)
    cache = paged(rng, 1, 1, 96, 2, 128)
    cache.table[0, 1] = -7
    before = cache.pool.clone()
    new = bd.cdsl_op_kvq_keep(cache, _ints([30]), _ints([[0, 3, 4, 40]]), _ints([4]))
    assert int(new) == 34
    # 33 -> 31 and 34 -> 32 lie on the missing page; 70 -> 33 too
    assert torch.equal(cache.pool, before)


def test_the_reference_codes_ties_to_even():
    code, e, none = coded(np.array([[0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5, 6] + [0.0] * 24]))
    assert code.reshape(-1)[:8].tolist() == [0, 2, 2, 4, 4, 6, 6, 7] and e.tolist() == [[0]] and not none.any()

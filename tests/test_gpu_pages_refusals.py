"""What the pages' bindings refuse before they call: tensors of another type, shape, order or device than the cache's.  Nothing is
launched and nothing changes."""
import pytest
import torch

pytestmark = pytest.mark.gpu

B, P, PAGES = 3, 4, 7


def _int(n, **kw):
    return torch.zeros(n, **{**dict(dtype=torch.int32, device="cuda"), **kw})


def _bad(n):
    """Tensors that are not n ints on the device, contiguous."""
    return {"short": _int(n - 1), "long": _int(n + 1), "two dims": _int((n, 1)), "int64": _int(n, dtype=torch.int64),
            "float": _int(n, dtype=torch.float32), "host": _int(n, device="cpu"), "every second": _int(2 * n)[::2]}


KINDS = ["short", "long", "two dims", "int64", "float", "host", "every second"]


def _cache():
    from paper_2412_10418_amd import binding as bd
    pool = bd.QuantCache.empty(2, PAGES, 1, 32, fmt="mxfp4").zero_()
    return bd.QuantCache(pool, torch.full((B, P), -1, dtype=torch.int32, device="cuda"), 32, "mxfp4")


@pytest.mark.parametrize("kind", KINDS)
def test_counts_of_the_pages(kind):
    from paper_2412_10418_amd import binding as bd
    c, refs, ints = _cache(), _bad(PAGES)[kind], _int(B)
    for call in (lambda: bd.cdsl_op_pages_fork(c, refs, ints), lambda: bd.cdsl_op_pages_reserve(c, refs, ints, ints, 5),
                 lambda: bd.cdsl_op_pages_free(c, refs, ints), lambda: bd.cdsl_op_pages_compact(c, refs)):
        with pytest.raises(ValueError):
            call()
    assert c.table.eq(-1).all() and not refs.any()


@pytest.mark.parametrize("kind", KINDS)
def test_numbers_of_the_prompts(kind):
    from paper_2412_10418_amd import binding as bd
    c, refs, bad, good = _cache(), _int(PAGES), _bad(B)[kind], _int(B) + 3
    for call in (lambda: bd.cdsl_op_pages_fork(c, refs, bad), lambda: bd.cdsl_op_pages_free(c, refs, bad),
                 lambda: bd.cdsl_op_pages_reserve(c, refs, bad, good, 5), lambda: bd.cdsl_op_pages_reserve(c, refs, good, bad, 5)):
        with pytest.raises(ValueError):
            call()
    assert c.table.eq(-1).all() and not refs.any()


@pytest.mark.parametrize("kind", KINDS)
def test_pages_to_copy(kind):
    from paper_2412_10418_amd import binding as bd
    c, other, bad, good = _cache(), _cache(), _bad(3)[kind], torch.arange(3, dtype=torch.int32, device="cuda")
    with pytest.raises(ValueError):
        bd.cdsl_op_pages_copy(c, good, other, bad)
    with pytest.raises(ValueError):
        bd.cdsl_op_pages_copy(c, bad, other, good)
    with pytest.raises(ValueError):
        bd.cdsl_op_pages_copy(c, good, other.pool, good)


def test_what_the_library_refuses_of_good_tensors():
    from paper_2412_10418_amd import binding as bd
    c, refs, ints = _cache(), _int(PAGES), _int(B)
    with pytest.raises(bd.CDSLError):
        bd.cdsl_op_pages_reserve(c, refs, ints, ints, -1)
    eight = bd.QuantCache(bd.QuantCache.empty(2, PAGES, 1, 32), c.table, 32, "int8")
    with pytest.raises(bd.CDSLError):
        bd.cdsl_op_pages_copy(c, ints, eight, ints)
    assert c.table.eq(-1).all() and not refs.any()

"""Sizes at the ends of their types in the calls around a drafted tree: refused on the host, without a GPU."""
import pytest

from test_tree_ops_host import _attend, _cache, _keep, _read, _write


def test_rows_beyond_the_launch_are_refused_before_they_are_planned():
    """Sizes whose products pass 32 and 64 bits: the plan divided by what was left of one."""
    from paper_2412_10418_amd import binding as bd
    c = _cache(batch=4096, n_kv_heads=1, head_dim=128)
    assert _attend(c, n=2 ** 30 - 1, H=1) == bd.CDSL_ERANGE
    assert _attend(_cache(batch=65535, n_kv_heads=1), n=2 ** 31 - 1, H=2 ** 31 - 1) == bd.CDSL_ERANGE


@pytest.mark.parametrize("args", [(2 ** 30 - 1, 4096, 1, 1, 128, 30000), (4096, 2 ** 30 - 1, 1, 1, 128, 0),
                                  (2 ** 31 - 1, 2 ** 31 - 1, 2 ** 31 - 1, 1, 128, 2 ** 31 - 1), (65536, 1, 1, 1, 64, 5000),
                                  (1, 2 ** 24, 1, 1, 64, 5000), (1, 1, 8, 8, 48, 30000)])
def test_no_workspace_for_what_is_refused(args):
    from paper_2412_10418_amd import binding as bd
    assert bd.lib().cdsl_op_tree_attention_workspace(*args) == 0


def test_pools_beyond_64_bits_have_no_size():
    """Their bytes came out modulo 2^64: 16896 for the first."""
    from paper_2412_10418_amd import binding as bd
    for layers, pages, heads in ((45078, 48912491, 32681), (1 << 20, 1 << 30, 1 << 6), (2 ** 31 - 1,) * 3):
        assert bd.lib().cdsl_op_kvq_pool_bytes(layers, pages, heads, 128) == 0
        c = _cache(n_layers=layers, pages=pages, n_kv_heads=heads, head_dim=128)
        assert _write(c) == _read(c) == _keep(c) == _attend(c, H=heads) == bd.CDSL_ERANGE
    assert bd.lib().cdsl_op_kvq_pool_bytes(1 << 10, 1 << 24, 1 << 10, 128) == 8448 << 44


def test_tables_end_where_positions_do():
    """The attention takes a position and the end of its page as an int: 2^26 pages of 32 tokens pass it."""
    from paper_2412_10418_amd import binding as bd
    for pages in (1 << 26, 2 ** 31 - 1):
        c = _cache(table_stride=pages)
        assert _write(c) == _read(c) == _keep(c) == _attend(c) == bd.CDSL_ERANGE
    c = _cache(table_stride=(1 << 26) - 1)
    assert _write(c, T=0) == _read(c, T=0) == _attend(c, n=0) == bd.CDSL_OK

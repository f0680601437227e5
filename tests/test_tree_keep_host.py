"""Refusals of the kept path's call, without a GPU."""
import pytest

from test_tree_ops_host import P, _cache, _keep

LENS, N_PATH, PATH = P, P + 0x100, P + 0x200      # 3 prompts, 4 nodes: 12, 12 and 48 bytes


@pytest.mark.parametrize("new", [LENS, LENS + 8, LENS - 8, N_PATH, N_PATH + 4, N_PATH - 8, PATH, PATH + 44, PATH - 8])
def test_new_lengths_over_what_the_call_reads(new):
    """The first layer's workgroups write them, the others' may read lens, n_path and path after that."""
    from paper_2412_10418_amd import binding as bd
    assert _keep(_cache(), lens=LENS, n_path=N_PATH, path=PATH, new=new) == bd.CDSL_EINVAL


def test_new_lengths_of_no_prompt():
    from paper_2412_10418_amd import binding as bd
    assert _keep(_cache(batch=0, table=None), lens=LENS, n_path=LENS, path=LENS, new=LENS) == bd.CDSL_OK

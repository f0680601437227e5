"""Lengths at the ends of their type in the kept path, target rows without mass in the verification, and caches whose
tensors are not to be exchanged."""
import numpy as np
import pytest
import torch

from test_gpu_tree_ops import _ints, _rows
from tree_ref import paged

pytestmark = pytest.mark.gpu


def test_new_lengths_at_the_ends_of_their_type():
    """They came out negative beyond 2^31 - 1, and the next call took that for an empty prompt.  Nothing moves there, nor
    does a length below 0, which counts as 0, move more than its path says."""
    from paper_2412_10418_amd import binding as bd
    rng = np.random.default_rng(81)
    cache = paged(rng, 2, 4, 64, 2, 64, "int8")
    x = _rows(rng, (4, 64, 2, 64), "f32")
    for layer in range(2):
        bd.cdsl_op_kvq_write(cache, x, -x, layer=layer)
    k, v = bd.cdsl_op_kvq_read(cache, 64)
    new = bd.cdsl_op_kvq_keep(cache, _ints([2 ** 31 - 1, 2 ** 31 - 3, -5, -(2 ** 31)]),
                              _ints([[0, 2, 3]] * 4), _ints([3, 3, 3, 0]))
    assert new.tolist() == [2 ** 31 - 1, 2 ** 31 - 1, 3, 0]
    for layer in range(2):
        k2, v2 = bd.cdsl_op_kvq_read(cache, 64, layer=layer)
        for old, got in ((k, k2), (v, v2)):
            want = old.clone()
            want[2, 1:3] = old[2, 2:4]
            assert torch.equal(got, want)


@pytest.mark.parametrize("replace", [True, False])
@pytest.mark.parametrize("V", [40, 20000, 40001])
def test_target_rows_without_mass(V, replace):
    """-1 where the walk ends at one without a child to test, argmax (the lowest id, 0) where one was rejected; so too at a
    node below the root."""
    from paper_2412_10418_amd import binding as bd
    p, q = np.zeros((4, 3, V), np.float32), np.full((4, 3, V), 1 / V, np.float32)
    p[2:, 0] = 1 / V                                      # node 1 is kept, node 2 is its child or a second one of the root
    parents = [[-1, -1, -1], [-1, 0, 0], [-1, 0, 0], [-1, 0, 1]]
    f = lambda x: torch.from_numpy(np.ascontiguousarray(x, np.float32)).cuda()  # noqa: E731
    path, m, tok = bd.cdsl_op_tree_accept(f(p), f(q), _ints([[0, 7, 8]] * 4), _ints(parents), f(np.full((4, 3), 0.5)),
                                          f(np.full(4, 0.5)), replace=replace)
    assert m.tolist() == [1, 1, 2, 2] and tok.tolist() == [-1, 0, -1, 0]
    assert path.tolist() == [[0, -1, -1], [0, -1, -1], [0, 1, -1], [0, 1, -1]]


def test_a_cache_keeps_its_tensors():
    """The library holds their addresses: another table put in the place of one had no effect on the calls."""
    cache = paged(np.random.default_rng(82), 1, 2, 40, 2, 32, "int8")
    for name in ("pool", "table", "head_dim", "fmt"):
        with pytest.raises(AttributeError):
            setattr(cache, name, getattr(cache, name))
    # what is written into the table counts
    from paper_2412_10418_amd import binding as bd
    x = _rows(np.random.default_rng(83), (2, 32, 2, 32), "f32")
    bd.cdsl_op_kvq_write(cache, x, -x)
    k, _ = bd.cdsl_op_kvq_read(cache, 32)
    cache.table.copy_(cache.table.flip(0))
    k2, _ = bd.cdsl_op_kvq_read(cache, 32)
    assert torch.equal(k2, k.flip(0))

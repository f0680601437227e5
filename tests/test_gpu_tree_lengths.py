"""Lengths at the ends of their type in the kept path."""
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

"""Forking tables with more columns than one launch has workgroups for, up to more entries than a launch may have threads."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("B,P", [(3, (1 << 18) + 1), (70, 600003), (256, (1 << 24) + 5)])
def test_fork_of_wide_tables(B, P):
    from paper_2412_10418_amd import binding as bd
    rng = np.random.default_rng([B, P])
    pages = 500
    cols = np.unique(np.concatenate([[0, 1, 3, 4, (1 << 18) - 1, 1 << 18, P - 1], rng.integers(0, P, 40)]))
    held = rng.integers(-1, pages, (B, len(cols)))
    table = torch.full((B, P), -1, dtype=torch.int32, device="cuda")
    at = torch.from_numpy(cols).cuda()
    table[:, at] = torch.from_numpy(held).int().cuda()
    cache = bd.QuantCache(bd.QuantCache.empty(1, pages, 1, 32, fmt="mxfp4"), table, 32, "mxfp4")
    refs = torch.from_numpy(np.bincount(held[held >= 0], minlength=pages)).int().cuda()
    parents = rng.integers(-1, B, B)
    bd.cdsl_op_pages_fork(cache, refs, torch.from_numpy(parents).int().cuda())
    want = np.where(parents[:, None] >= 0, held[parents], -1)
    assert np.array_equal(table[:, at].cpu().numpy(), want)
    assert sum(int((row != -1).sum()) for row in table) == int((want != -1).sum())
    assert np.array_equal(refs.cpu().numpy(), np.bincount(want[want >= 0], minlength=pages))

"""Workspaces of the attention over the 4-bit cache that are there but too small: refused on the host, before a launch."""
import pytest

from test_tree_ops_host import P, _attend, _cache

# B, n, H, KV heads, head dim, longest: keys that are split over several workgroups, of each kernel
SPLIT = [(3, 1, 8, 4, 64, 30000), (1, 6, 8, 2, 128, 5000), (1, 40, 8, 2, 128, 9000), (8, 17, 32, 8, 128, 6600), (8, 65, 32, 8, 128, 8192)]


@pytest.mark.parametrize("dtype", [0, 1], ids=["f32", "bf16"])
@pytest.mark.parametrize("case", SPLIT, ids=str)
def test_a_workspace_that_is_too_small(case, dtype):
    from paper_2412_10418_amd import binding as bd
    B, n, H, heads, hd, longest = case
    c = _cache(format=4, batch=B, n_kv_heads=heads, head_dim=hd, table_stride=1000)
    one = 4 * n * H * (hd + 2)        # bytes of a part of a prompt's keys: a sum, a maximum and a result per row
    assert bd.lib().cdsl_op_tree_attention_workspace(B, n, H, heads, hd, longest) >= (B + 1) * one
    for n_bytes in (0, 1, 16, one, B * one, (B + 1) * one - 1):
        assert _attend(c, dtype=dtype, n=n, H=H, max_len=longest, ws=P, ws_bytes=n_bytes) == bd.CDSL_EINVAL, n_bytes
    assert _attend(c, dtype=dtype, n=n, H=H, max_len=longest, ws=None, ws_bytes=1 << 40) == bd.CDSL_EINVAL
    assert _attend(c, dtype=dtype, n=n, H=H, max_len=longest, ws=P + 8, ws_bytes=1 << 40) == bd.CDSL_EINVAL

"""Plain 64-bit forms of the 4-bit cache, for its tests: what rows read back as, where a token's bytes stand in a unit, and
a cache over pages in no order.  (Attention over it: tree_ref.py, on the rows that are read back.)"""
import numpy as np
import torch

GRID = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6])


def coded(x):
    """(codes 0..15, exponents of the scales, which rows are NaN) of rows x [..., hd]: the nearest of the grid by distance, of
    two as near the one with the even code."""
    x = np.asarray(x, np.float64)
    none = ~np.isfinite(x).all(-1)
    b = np.where(none[..., None], 0, x).reshape(*x.shape[:-1], x.shape[-1] // 32, 32)
    a = np.abs(b).max(-1)
    e = np.full(a.shape, -125)
    for k in range(-125, 126):          # the smallest power with a <= 6 s
        e = np.where((a > 6 * 2.0 ** (k - 1)) & (k <= 125), k, e)
    far = np.abs(np.abs(b / 2.0 ** e[..., None])[..., None] - GRID)
    return _nearest(far) + 8 * np.signbit(b), e, none


def _nearest(far):
    best = far.min(-1, keepdims=True)
    tie = far == best
    first = tie.argmax(-1)
    last = 7 - tie[..., ::-1].argmax(-1)
    return np.where(first % 2 == 0, first, last)


def quantised(x):
    """What rows x [..., hd] read back as, in fp32."""
    code, e, none = coded(x)
    y = np.where(code < 8, 1, -1) * GRID[code % 8] * 2.0 ** e[..., None]
    y = y.reshape(np.shape(x)).astype(np.float32)
    return np.where(none[..., None], np.float32(np.nan), y)


def places(hd):
    """[32, hd + hd / 16] byte offsets of a slot's key codes, value codes, key scales and value scales."""
    out = np.zeros((32, hd + hd // 16), np.int64)
    W = 2 if hd > 32 else 1
    for s in range(32):
        at = []
        for d in range(0, hd, 2):
            at.append(d // 64 * 1024 + (d % 32 // 8 * 16 + s % 16) * 8 * W + d // 32 % 2 * 8 + s // 16 * 4 + d % 8 // 2)
        for d in range(0, hd, 2):
            at.append(16 * hd + d // 64 * 1024 + (s % 16 // 4 * 16 + d % 32 // 2) * 8 * W + d // 32 % 2 * 8 + s // 16 * 4 + s % 4)
        for d in range(0, hd, 32):
            at.append(32 * hd + d // 64 * 64 + s % 16 * 2 * W + d // 32 % 2 * 2 + s // 16)
        for d in range(0, hd, 32):
            at.append(33 * hd + d // 64 * 64 + s % 16 // 4 * 8 * W + d // 32 % 2 * 8 + s // 16 * 4 + s % 4)
        out[s] = at
    return out


def token_bytes(k, v):
    """The bytes of tokens k, v [..., hd], in the order of places()."""
    out = []
    for x in (k, v):
        code, e, none = coded(x)
        code = np.where(none[..., None], 0, code.reshape(np.shape(x)))
        out.append(((code[..., 0::2] | code[..., 1::2] << 4).astype(np.uint8), np.where(none[..., None], 255, e + 127).astype(np.uint8)))
    return np.concatenate([out[0][0], out[1][0], out[0][1], out[1][1]], -1)


def paged(rng, layers, B, tokens, heads, hd, spare=2, fill=None):
    """A 4-bit QuantCache whose pages hold leftovers, in no order."""
    from paper_2412_10418_amd.binding import QuantCache
    per = -(-tokens // 32)
    pages = B * per + spare
    pool = QuantCache.empty(layers, pages, heads, hd, fmt="mxfp4")
    if fill is None:
        pool.copy_(torch.from_numpy(rng.integers(0, 256, pool.shape, dtype=np.uint8)))
    else:
        pool.fill_(fill)
    table = torch.from_numpy(rng.permutation(pages)[:B * per].reshape(B, per).astype(np.int32)).cuda()
    return QuantCache(pool, table, hd, "mxfp4")
